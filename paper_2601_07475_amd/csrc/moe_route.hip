// The router of a mixture of experts: scores of all experts for a token, its best ones and their weights.
//   l[m, e] = sum_k x[m, k] r[e, k];   s = softmax(l) or 1 / (1 + exp(-l));   best by s (+ bias);   weights: their s, or their shares of those
// Which experts are best is decided by sums in 64 bits of exact products: near ties fall as the definition has it down to the roundings of such a sum, whose order differs
// between the kernels, and not as an order of fp32 sums does.
//
// One launch where a workgroup a token gets through the router's weights quickly; otherwise scores_kernel, on v_mfma_f64_16x16x4_f64, leaves sums of runs of K
// in the workspace and choose_kernel adds them up in their order.  Bound by two launches for a few tokens, by the 64-bit matrix rate for many (2 M K E of
// 78 * 10^12 a second).
// Measured, us a call: 1 x 4096, two of eight 5.9 to 6.2 (one launch: a trip to memory for x and the weights, the sums of 16 waves, two choices one after the other);
// 64 x 8192, eight of 256 15.3 (a workgroup a token, which reads all 4 MB of the weights for each, 119).
#include "internal.h"

#include <algorithm>

namespace arcq {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef double double4v __attribute__((ext_vector_type(4)));

struct RouteArgs {
    const _Float16 *x, *router;
    int64_t ldx, ldr;
    const float* bias;
    int M, K, E, top;
    uint32_t flags;
    int32_t* ids;
    float* weights;
    double* sums;                               // [splits][M][E]
    int splits;
};

// A value's neighbour by a data-parallel move (row shifts, then the last lane of a row, of two rows, to the next): lanes without one get `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v, double none) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v), o = __builtin_bit_cast(uint64_t, none);
    const uint32_t lo = __builtin_amdgcn_update_dpp((int)(uint32_t)o, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp((int)(uint32_t)(o >> 32), (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double last_lane(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <typename Op>
__device__ __forceinline__ double over_wave(double v, double none, const Op& op) {
    v = op(v, moved<0x111, 0xF>(v, none));      // row_shr 1, 2, 4, 8
    v = op(v, moved<0x112, 0xF>(v, none));
    v = op(v, moved<0x114, 0xF>(v, none));
    v = op(v, moved<0x118, 0xF>(v, none));
    v = op(v, moved<0x142, 0xA>(v, none));      // row_bcast 15 into rows 1 and 3, row_bcast 31 into rows 2 and 3
    v = op(v, moved<0x143, 0xC>(v, none));
    return last_lane(v);
}
__device__ __forceinline__ double wave_sum(double v) {
    return over_wave(v, 0.0, [](double a, double b) { return a + b; });
}
// (what is not a number is passed over)
__device__ __forceinline__ double wave_max(double v) {
    return over_wave(v, -INFINITY, [](double a, double b) { return fmax(a, b); });
}

// One wave: the best experts of token m by its scores; logits[j]: of expert 64 j + lane, not a number past the last one.
template <int PER>
__device__ __forceinline__ void choose(const double (&logits)[PER], const RouteArgs& a, int64_t m) {
    const int lane = threadIdx.x & 63;
    const bool sigmoid = (a.flags & ARCQ_MOE_SIGMOID) != 0;
    double score[PER], rank[PER];
    double most = -INFINITY;
#pragma unroll
    for (int j = 0; j < PER; ++j) most = fmax(most, logits[j]);
    most = wave_max(most);
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        score[j] = sigmoid ? 1.0 / (1.0 + exp(-logits[j])) : exp(logits[j] - most);
        if (64 * j + lane < a.E) sum += score[j];
    }
    sum = sigmoid ? 1.0 : wave_sum(sum);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = 64 * j + lane;
        score[j] /= sum;
        rank[j] = a.bias && e < a.E ? score[j] + (double)a.bias[e] : logits[j];
    }
    double chosen = 0.0, mine = 0.0;
    int32_t id = -1;
    for (int t = 0; t < a.top; ++t) {
        double best = -INFINITY;
#pragma unroll
        for (int j = 0; j < PER; ++j) best = fmax(best, rank[j]);       // (passes over what is taken)
        best = wave_max(best);
        int e = -1;
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint64_t equal = __ballot(rank[j] == best);
            if (e < 0 && equal != 0) {
                const int at = (int)__builtin_ctzll(equal);
                const uint64_t b = __builtin_bit_cast(uint64_t, score[j]);
                const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, at), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), at);
                e = 64 * j + at;
                s = __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
                if (lane == at) rank[j] = __builtin_nan("");
            }
        }
        chosen += s;
        if (lane == t) id = e, mine = s;
    }
    if (lane < a.top) {
        a.ids[m * a.top + lane] = id;
        a.weights[m * a.top + lane] = (float)(a.flags & ARCQ_MOE_RENORMALIZE ? mine / chosen : mine);
    }
}

// A workgroup a token, its 16 waves in teams of `team` for an expert.
template <int PER>
__global__ __launch_bounds__(1024) void route_token_kernel(RouteArgs a, int team) {
    __shared__ double part[16][64 * PER];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), run = wave % team;
    const int64_t m = blockIdx.x;
    const _Float16* x = a.x + m * a.ldx;
    for (int e = wave / team; e < a.E; e += 16 / team) {
        const _Float16* r = a.router + e * a.ldr;
        double sum = 0.0;
        for (int k = 8 * (64 * run + lane); k < a.K; k += 512 * team) {
            const half8 u = *reinterpret_cast<const half8*>(x + k), v = *reinterpret_cast<const half8*>(r + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)((float)u[i] * (float)v[i]);
        }
        sum = wave_sum(sum);
        if (lane == 0) part[run][e] = sum;
    }
    __syncthreads();
    if (wave != 0) return;
    double logits[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = 64 * j + lane;
        logits[j] = __builtin_nan("");
        if (e < a.E) {
            logits[j] = part[0][e];
            for (int w = 1; w < team; ++w) logits[j] += part[w][e];
        }
    }
    choose<PER>(logits, a, m);
}

// 16 tokens by 16 experts, one of `splits` runs of K, in four waves.  Lane (i, q) brings k = 32 c + 8 q .. + 7 of token i and of expert i: the s-th of
// these of the four lane groups are a step of the matrix instruction.
__global__ __launch_bounds__(256) void scores_kernel(RouteArgs a, uint32_t tiles_e) {
    __shared__ double part[4][256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    const uint32_t tile = blockIdx.x / (uint32_t)a.splits, split = blockIdx.x % (uint32_t)a.splits;
    const int m0 = 16 * (int)(tile / tiles_e), e0 = 16 * (int)(tile % tiles_e);
    const _Float16* x = a.x + (int64_t)min(m0 + i, a.M - 1) * a.ldx;
    const _Float16* r = a.router + (int64_t)min(e0 + i, a.E - 1) * a.ldr;
    const int chunks = (a.K + 31) >> 5, runs = 4 * a.splits, run = 4 * (int)split + wave;
    const int c0 = (int)((int64_t)run * chunks / runs), c1 = (int)((int64_t)(run + 1) * chunks / runs);
    double4v acc = {0.0, 0.0, 0.0, 0.0};
    constexpr int G = 4;                            // chunks asked for at once
    for (int c = c0; c < c1; c += G) {
        half8 u[G], v[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {               // (past the end: the last chunk again; pieces past the end of a row, its last one: counted as zeros)
            const int k = min(32 * min(c + g, c1 - 1) + 8 * q, a.K - 8);
            u[g] = *reinterpret_cast<const half8*>(x + k);
            v[g] = *reinterpret_cast<const half8*>(r + k);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (c + g >= c1) break;
            if (32 * (c + g) + 8 * q >= a.K) u[g] = half8{0, 0, 0, 0, 0, 0, 0, 0}, v[g] = u[g];
#pragma unroll
            for (int s = 0; s < 8; ++s) acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(float)u[g][s], (double)(float)v[g][s], acc, 0, 0, 0);
        }
    }
    // a lane has the sums of expert i and tokens q, q + 4, q + 8, q + 12
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][16 * (4 * k + q) + i] = acc[k];
    __syncthreads();
    const int m = m0 + (tid >> 4), e = e0 + (tid & 15);
    if (m < a.M && e < a.E) a.sums[((int64_t)split * a.M + m) * a.E + e] = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
}

// A wave a token.
template <int PER>
__global__ __launch_bounds__(256) void choose_kernel(RouteArgs a) {
    const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (m >= a.M) return;
    const int lane = threadIdx.x & 63;
    double logits[PER];
    constexpr int G = PER < 4 ? 8 : PER < 16 ? 4 : 2;       // runs asked for at once
    const double* at = a.sums + m * a.E;
#pragma unroll
    for (int j = 0; j < PER; ++j) logits[j] = 0.0;
    for (int s = 0; s < a.splits; s += G) {
        double v[G][PER];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < PER; ++j) v[g][j] = at[(int64_t)min(s + g, a.splits - 1) * a.M * a.E + min(64 * j + lane, a.E - 1)];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < PER; ++j) logits[j] += s + g < a.splits ? v[g][j] : 0.0;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (64 * j + lane >= a.E) logits[j] = __builtin_nan("");
    choose<PER>(logits, a, m);
}

// Tokens of a launch: the workspace and grids stay within bounds for any number of them.
constexpr int64_t kMostTokens = 4096;

// Whether a workgroup a token is quickest: it reads all of the router's weights by itself, 128 KB at most.  Measured, us a call, and the other way:
// 8 experts, K = 4096, 1 to 256 tokens 6.5, 9.3; 60 and 1024 6.6, 9.3; 60 and 4096 13 to 14, 9.2.
bool by_token(int64_t K, int64_t E) { return E <= 64 && K * E <= 65536; }

// Runs of K: two workgroups a compute unit, with four chunks of 32 for each wave.
constexpr int64_t kRunWorkgroups = 2 * 256, kRunK = 512;
int splits_of(int64_t M, int64_t K, int64_t E) {
    const int64_t tiles = (M + 15) / 16 * ((E + 15) / 16);
    return (int)std::max<int64_t>(1, std::min<int64_t>(kRunWorkgroups / tiles, K / kRunK));
}

template <int PER>
arcq_status launch_choose(const RouteArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL(choose_kernel<PER>, dim3((unsigned)((a.M + 3) / 4)), dim3(256), 0, stream, a);
    return check_launch("choose_kernel");
}

}  // namespace

// Fewer tokens may go in more runs and need more room than more tokens do, so this is the most that any number of them up to M needs: for every number of
// runs, as many tokens as still go in that many.
size_t moe_route_workspace_bytes(int64_t M, int64_t K, int64_t E) {
    if (by_token(K, E)) return 0;
    M = std::min(M, kMostTokens);
    const int64_t tiles_e = (E + 15) / 16;
    int64_t rows = M;                               // in one run
    for (int64_t runs = 2; runs <= K / kRunK && runs * tiles_e <= kRunWorkgroups; ++runs) rows = std::max(rows, runs * std::min(M, kRunWorkgroups / (runs * tiles_e) * 16));
    return (size_t)rows * (size_t)E * sizeof(double);
}

arcq_status launch_moe_route(const void* x, int64_t M, int64_t K, int64_t ldx, const void* router, int64_t ldr, int64_t E, const float* bias, int64_t top,
                             uint32_t flags, int32_t* ids, float* weights, void* workspace, hipStream_t stream) {
    const int splits = splits_of(std::min(M, kMostTokens), K, E);       // (a last launch of fewer tokens has the runs of the first: there is room for those)
    for (int64_t m = 0; m < M; m += kMostTokens) {
        const int64_t rows = std::min(M - m, kMostTokens);
        const RouteArgs a = {static_cast<const _Float16*>(x) + m * ldx, static_cast<const _Float16*>(router), ldx, ldr, bias, (int)rows, (int)K, (int)E, (int)top, flags,
                             ids + m * top, weights + m * top, static_cast<double*>(workspace), splits};
        if (by_token(K, E)) {
            int team = 1;
            while (2 * team * E <= 16 && 1024 * team <= K) team *= 2;
            hipLaunchKernelGGL(route_token_kernel<1>, dim3((unsigned)rows), dim3(1024), 0, stream, a, team);
            if (arcq_status st = check_launch("route_token_kernel")) return st;
            continue;
        }
        const unsigned tiles_e = (unsigned)((E + 15) / 16), tiles_m = (unsigned)((rows + 15) / 16);
        hipLaunchKernelGGL(scores_kernel, dim3(tiles_e * tiles_m * (unsigned)splits), dim3(256), 0, stream, a, tiles_e);
        if (arcq_status st = check_launch("scores_kernel")) return st;
        const arcq_status st = E <= 64    ? launch_choose<1>(a, stream)
                               : E <= 128 ? launch_choose<2>(a, stream)
                               : E <= 256 ? launch_choose<4>(a, stream)
                               : E <= 512 ? launch_choose<8>(a, stream)
                                          : launch_choose<16>(a, stream);
        if (st) return st;
    }
    return ARCQ_OK;
}

}  // namespace arcq
