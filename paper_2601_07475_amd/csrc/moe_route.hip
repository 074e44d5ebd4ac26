// The router of a mixture of experts: scores of all experts for a token, its best ones and their weights.
//   l[m, e] = sum_k x[m, k] r[e, k];   s = softmax(l) or 1 / (1 + exp(-l));   best by s (+ bias);   weights: their s, or their shares of those
// Which experts are best is decided by sums in 64 bits of exact products, so near ties fall as the definition has it and not as an order of fp32 sums does.
#include "internal.h"

#include <algorithm>

namespace arcq {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
constexpr int kPerLane = ARCQ_MOE_MAX_EXPERTS / 64;

struct RouteArgs {
    const _Float16 *x, *router;
    int64_t ldx, ldr;
    const float* bias;
    int M, K, E, top;
    uint32_t flags;
    int32_t* ids;
    float* weights;
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}

// One wave: the best experts of a token by its scores, in LDS.
__device__ void choose(const double* logits, const RouteArgs& a, int64_t m) {
    const int lane = threadIdx.x & 63;
    const bool sigmoid = (a.flags & ARCQ_MOE_SIGMOID) != 0;
    double score[kPerLane], rank[kPerLane];
    double most = -INFINITY;
    for (int j = 0; j < kPerLane; ++j) {
        const int e = 64 * j + lane;
        score[j] = e < a.E ? logits[e] : __builtin_nan("");
        most = fmax(most, score[j]);
    }
    most = wave_max(most);
    double sum = 0.0;
    for (int j = 0; j < kPerLane; ++j) {
        rank[j] = score[j];
        if (64 * j + lane < a.E) {
            score[j] = sigmoid ? 1.0 / (1.0 + exp(-score[j])) : exp(score[j] - most);
            sum += score[j];
        }
    }
    sum = sigmoid ? 1.0 : wave_sum(sum);
    for (int j = 0; j < kPerLane; ++j) {
        score[j] /= sum;
        if (a.bias && 64 * j + lane < a.E) rank[j] = score[j] + (double)a.bias[64 * j + lane];
    }
    double chosen = 0.0, mine = 0.0;
    int32_t id = -1;
    for (int t = 0; t < a.top; ++t) {
        double best = -INFINITY;
        for (int j = 0; j < kPerLane; ++j) best = fmax(best, rank[j]);     // (fmax passes over what is not a number: taken, or no expert)
        best = wave_max(best);
        int e = -1;
        double s = 0.0;
        for (int j = 0; j < kPerLane; ++j) {
            const uint64_t equal = __ballot(rank[j] == best);
            if (e < 0 && equal != 0) {
                const int at = __builtin_ctzll(equal);
                e = 64 * j + at;
                s = __shfl(score[j], at);
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

// A workgroup a token.
__global__ __launch_bounds__(1024) void route_token_kernel(RouteArgs a) {
    __shared__ double logits[ARCQ_MOE_MAX_EXPERTS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m = blockIdx.x;
    const _Float16* x = a.x + m * a.ldx;
    for (int e = wave; e < a.E; e += 16) {
        const _Float16* r = a.router + e * a.ldr;
        double sum = 0.0;
        for (int k = 8 * lane; k < a.K; k += 512) {
            const half8 u = *reinterpret_cast<const half8*>(x + k), v = *reinterpret_cast<const half8*>(r + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)((float)u[i] * (float)v[i]);
        }
        sum = wave_sum(sum);
        if (lane == 0) logits[e] = sum;
    }
    __syncthreads();
    if (wave == 0) choose(logits, a, m);
}

}  // namespace

size_t moe_route_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

arcq_status launch_moe_route(const void* x, int64_t M, int64_t K, int64_t ldx, const void* router, int64_t ldr, int64_t E, const float* bias, int64_t top,
                             uint32_t flags, int32_t* ids, float* weights, void*, hipStream_t stream) {
    const RouteArgs a = {static_cast<const _Float16*>(x), static_cast<const _Float16*>(router), ldx, ldr, bias, (int)M, (int)K, (int)E, (int)top, flags, ids, weights};
    hipLaunchKernelGGL(route_token_kernel, dim3((unsigned)M), dim3(1024), 0, stream, a);
    return check_launch("route_token_kernel");
}

}  // namespace arcq
