// The experts of a mixture for a few tokens, on packed 4-bit weights, as two kernels:
//   h[m, j] = w[m, j] act(x[m] G_e^T) (x[m] U_e^T)        e = ids[m, j]            up_kernel
//   y[m]    = sum_j h[m, j] D_e^T + residual[m]                                    down_kernel
// x fp16, G over U the 2 I rows of an expert's first operand, D its second; NVFP4 (B = 16) or MXFP4 (B = 32).
//
// Bound by reading the chosen experts' weights once (3 K I weights each, 9/16 or 17/32 byte a weight).  Tokens are a row tile of v_mfma_f32_16x16x32_f16, so
// up to 16 (8 behind the activation) cost what one does.
//
// Every workgroup finds out by itself which tokens choose an expert (lists_of): no kernel in front, and none that waits for the host.  An expert that a token
// names twice counts once, with both weights: lists then hold a token once, and sums do not depend on the order of a list.
//
// h is held as two fp16 numbers, h / 16 rounded and 2^11 times what that leaves: 22 bits of h down to 2^-10, 2^-32 below it, up to 2^20.  (One fp16 number would put
// its rounding, 2^-12, behind an fp32 y.)  The two are rows i and i + 8 of one row tile, so the second costs no more matrix instructions than the tile's
// free rows; the halves of a wave hold the sums of either and are put together when a wave is done with an expert.
//
// down_kernel's reduction runs over all chosen experts' channels one after the other, in equal shares for the waves of a workgroup; a wave adds what it has of an
// expert to its own sums of all tokens in LDS, and the waves' sums are added in their order at the end.  No atomics: the same inputs give the same bits.
#include "epilogue.h"
#include "internal.h"
#include "lds_dma.h"
#include "row_products.h"

#include <algorithm>
#include <type_traits>

namespace arcq {

namespace {

constexpr int kMostExperts = ARCQ_MOE_MAX_EXPERTS, kMostTokens = 64, kMostSlots = kMostTokens * ARCQ_MOE_MAX_TOP_K;     // of a launch
constexpr float kLow = 0x1p-11f;                // what the second number of h counts
constexpr float kUnit = 16.0f;                  // what the first one counts

struct Experts {
    const uint8_t *codes, *scales;              // [E, rows, pitch]
    const float* tensor_scales;                 // NVFP4: [E]
    int64_t code_pitch, scale_pitch;            // bytes of a row
    int rows;                                   // of an expert
};

// Which slots (token, choice) every expert has.
struct Lists {
    int start[kMostExperts + 1], count[kMostExperts];
    int active[kMostExperts];                   // experts with slots, ascending
    int slots[kMostSlots];
    int actives;
};

// All threads of the workgroup.  ids outside 0 .. E - 1: no expert.
template <int THREADS>
__device__ void lists_of(const int32_t* __restrict__ ids, int M, int top, int E, Lists& l) {
    const int tid = threadIdx.x, slots = M * top;
    constexpr int PER = (kMostSlots + THREADS - 1) / THREADS;
    int id[PER], at[PER];
    for (int e = tid; e < E; e += THREADS) l.count[e] = 0;
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = tid + p * THREADS;
        id[p] = -1;
        if (t < slots) {
            const int e = ids[t], first = t - t % top;
            bool fresh = e >= 0 && e < E;
            for (int u = first; u < t; ++u) fresh = fresh && ids[u] != e;       // (a later choice of the same expert counts with the first)
            if (fresh) {
                id[p] = e;
                at[p] = atomicAdd(&l.count[e], 1);
            }
        }
    }
    __syncthreads();
    if (tid < 64) {
        int begin = 0, actives = 0;
        for (int base = 0; base < E; base += 64) {
            const int e = base + tid, n = e < E ? l.count[e] : 0;
            int sum = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(sum, d);
                if (tid >= d) sum += other;
            }
            const uint64_t some = __ballot(n > 0);
            if (e < E) l.start[e] = begin + sum - n;
            if (n > 0) l.active[actives + __popcll(some & ((1ull << tid) - 1ull))] = e;
            begin += __shfl(sum, 63);
            actives += __popcll(some);
        }
        if (tid == 0) l.actives = actives;
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PER; ++p)
        if (id[p] >= 0) l.slots[l.start[id[p]] + at[p]] = tid + p * THREADS;
    __syncthreads();
}

// A wave's product of up to 16 MT rows (fragments from `row`, where `valid`) with NT tiles of 16 weight rows (this lane's: wc, ws) over chunks c0 .. c1 - 1
// of 128 k, the last of which may be the part behind the last whole one of K.
template <int B, int MT, int NT>
__device__ __forceinline__ void accumulate(const uint16_t* const (&row)[MT], const bool (&valid)[MT], const uint8_t* const (&wc)[NT], const uint8_t* const (&ws)[NT],
                                           int K, int c0, int c1, float4v (&acc)[1][MT][NT]) {
    constexpr int SB = 128 / B, G = MT == 1 ? 4 : MT == 2 ? 2 : 1;     // scale bytes of a chunk; chunks in flight
    const int lane = threadIdx.x & 63, q = lane >> 4;
    const int whole = min(c1, K >> 7);
    for (int c = c0; c < whole; c += G) {
        const int count = min(G, whole - c);
        u32x2 sc[NT];
        u32x4 cw[G][NT];
        half8 xf[G][MT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t at = (int64_t)SB * (c + min(q, count - 1));
            if constexpr (B == 16) {
                const uint2 v = load8_a1(ws[t] + at);
                sc[t] = u32x2{v.x, v.y};
            } else {
                sc[t] = u32x2{load4_a1(ws[t] + at), 0u};
            }
        }
#pragma unroll
        for (int d = 0; d < G; ++d)
            if (d < count)
#pragma unroll
                for (int t = 0; t < NT; ++t) cw[d][t] = *reinterpret_cast<const u32x4_a4*>(wc[t] + 64 * (int64_t)(c + d) + 16 * q);
#pragma unroll
        for (int r = 0; r < MT; ++r) {
#pragma unroll
            for (int d = 0; d < G; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[d][r][j] = half8{0, 0, 0, 0, 0, 0, 0, 0};
            if (valid[r]) {
#pragma unroll
                for (int d = 0; d < G; ++d)
                    if (d < count)
#pragma unroll
                        for (int j = 0; j < 4; ++j) xf[d][r][j] = *reinterpret_cast<const half8*>(row[r] + 128 * (c + d) + 32 * j + 8 * q);
            }
        }
        uint32_t sw[4][NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint32_t s[4];
            scales_of_group<B>(make_uint2(sc[t][0], sc[t][1]), s);
#pragma unroll
            for (int d = 0; d < 4; ++d) sw[d][t] = s[d];
        }
#pragma unroll
        for (int d = 0; d < G; ++d) {
            if (d < count) {
                uint4 words[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) words[t] = make_uint4(cw[d][t][0], cw[d][t][1], cw[d][t][2], cw[d][t][3]);
                multiply_chunk<B, MT, NT, 1>(xf[d], words, sw[d], acc);
            }
        }
    }
    if (c1 > whole && c0 < c1) {                        // less than a chunk: blocks past the end count as zero codes, rows are read from their start there
        const int c = K >> 7, blocks = K / B, pieces = K >> 3;
        const int b0 = B == 16 ? 8 * c + 2 * q : 4 * c + q;
        uint4 words[NT];
        uint32_t sw[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (B == 16) {
                const uint2 lo = load8_a8(wc[t] + 8 * (int64_t)min(b0, blocks - 1)), hi = load8_a8(wc[t] + 8 * (int64_t)min(b0 + 1, blocks - 1));
                const bool ok0 = b0 < blocks, ok1 = b0 + 1 < blocks;
                words[t] = make_uint4(ok0 ? lo.x : 0, ok0 ? lo.y : 0, ok1 ? hi.x : 0, ok1 ? hi.y : 0);
            } else {
                const uint4 v = load16_a4(wc[t] + 16 * (int64_t)min(b0, blocks - 1));
                const bool ok = b0 < blocks;
                words[t] = make_uint4(ok ? v.x : 0, ok ? v.y : 0, ok ? v.z : 0, ok ? v.w : 0);
            }
            sw[t] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sw[t] |= (uint32_t)ws[t][min(B == 16 ? 8 * c + 2 * j + (q >> 1) : 4 * c + j, blocks - 1)] << (8 * j);
        }
        half8 xf[MT][4];
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int piece = 16 * c + 4 * j + q;
                xf[r][j] = half8{0, 0, 0, 0, 0, 0, 0, 0};
                if (valid[r] && piece < pieces) xf[r][j] = *reinterpret_cast<const half8*>(row[r] + 8 * piece);
            }
        multiply_chunk<B, MT, NT, 1>(xf, words, sw, acc);
    }
}

template <int MT, int NT>
__device__ __forceinline__ void clear(float4v (&acc)[1][MT][NT]) {
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[0][r][t] = float4v{0.f, 0.f, 0.f, 0.f};
}

struct UpArgs {
    const uint16_t* x;
    int64_t ldx;
    const int32_t* ids;
    const float* weights;
    int M, top, E, K, I, activation;
    Experts up;
    uint16_t *high, *low;                       // [M top, I]
    int tiles;
};

// A workgroup: 16 columns of one expert, that is 16 rows of G and of U, K split over the waves, tokens 32 (16) at a time.
template <int B, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 4))) void up_kernel(UpArgs a) {
    constexpr int THREADS = 64 * WAVES;
    __shared__ Lists l;
    __shared__ float red[WAVES][2][2][4][64];       // row tile, G or U, element, lane
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15;
    lists_of<THREADS>(a.ids, a.M, a.top, a.E, l);
    const int nth = (int)(blockIdx.x / (uint32_t)a.tiles), n0 = 16 * (int)(blockIdx.x % (uint32_t)a.tiles);
    if (nth >= l.actives) return;
    const int e = __builtin_amdgcn_readfirstlane(l.active[nth]), count = __builtin_amdgcn_readfirstlane(l.count[e]), first = __builtin_amdgcn_readfirstlane(l.start[e]);
    const float alpha = B == 16 ? a.up.tensor_scales[e] : 1.0f;
    const uint8_t *wc[2], *ws[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t at = (int64_t)e * a.up.rows + t * a.I + n0 + i;   // (I is a multiple of 16)
        wc[t] = a.up.codes + at * a.up.code_pitch;
        ws[t] = a.up.scales + at * a.up.scale_pitch;
    }
    const int chunks = (a.K + 127) >> 7, c0 = wave * chunks / WAVES, c1 = (wave + 1) * chunks / WAVES;
    auto tokens = [&](auto mt_tag, int r0) {
        constexpr int MT = decltype(mt_tag)::value;
        const uint16_t* row[MT];
        bool valid[MT];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            valid[r] = r0 + 16 * r + i < count;
            row[r] = a.x + (int64_t)(l.slots[first + min(r0 + 16 * r + i, count - 1)] / a.top) * a.ldx;
        }
        float4v acc[1][MT][2];
        clear<MT, 2>(acc);
        accumulate<B, MT, 2>(row, valid, wc, ws, a.K, c0, c1, acc);
        if (r0 > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) red[wave][r][t][k][lane] = acc[0][r][t][k];
        __syncthreads();
        for (int idx = tid; idx < MT * 256; idx += THREADS) {
            const int r = idx >> 8, k = (idx >> 6) & 3, at = idx & 63, which = r0 + 16 * r + 4 * (at >> 4) + k;
            if (which >= count) continue;
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) g += red[w][r][0][k][at], u += red[w][r][1][k][at];
            float v[1] = {g * alpha};
            activate(v, a.activation);
            const int slot = l.slots[first + which];
            float weight = a.weights[slot];
            for (int s = slot + 1; s % a.top != 0; ++s)                  // the same expert again
                if (a.ids[s] == e) weight += a.weights[s];
            const float h = v[0] * (u * alpha) * weight * (1.0f / kUnit);
            const _Float16 high = (_Float16)h, low = (_Float16)((h - (float)high) * (1.0f / kLow));
            const int64_t to = (int64_t)slot * a.I + n0 + (at & 15);
            a.high[to] = __builtin_bit_cast(uint16_t, high);
            a.low[to] = __builtin_bit_cast(uint16_t, low);
        }
    };
    for (int r0 = 0; r0 < count; r0 += 32) {
        if (count - r0 <= 16) tokens(std::integral_constant<int, 1>{}, r0);
        else tokens(std::integral_constant<int, 2>{}, r0);
    }
}

template <typename OutT>
struct DownArgs {
    const uint16_t *high, *low;
    const int32_t* ids;
    int M, top, E, I, N;
    Experts down;
    const OutT* residual;
    int64_t ldr;
    OutT* y;
    int64_t ldy;
};

// A workgroup: 16 NT columns of y for all tokens.
template <int B, int NT, int WAVES, typename OutT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 4))) void down_kernel(DownArgs<OutT> a) {
    constexpr int THREADS = 64 * WAVES, COLS = 16 * NT;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Lists& l = *reinterpret_cast<Lists*>(lds);
    float* sums = reinterpret_cast<float*>(lds + sizeof(Lists));        // [WAVES][M][COLS]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    for (int k = tid; k < WAVES * a.M * COLS; k += THREADS) sums[k] = 0.0f;
    lists_of<THREADS>(a.ids, a.M, a.top, a.E, l);
    float* own = sums + wave * a.M * COLS;
    const int n0 = (int)blockIdx.x * COLS;
    const int per = (a.I + 127) >> 7, all = __builtin_amdgcn_readfirstlane(l.actives) * per;
    const int end = (int)((int64_t)(wave + 1) * all / WAVES);
    for (int c = (int)((int64_t)wave * all / WAVES); c < end;) {
        const int nth = c / per, c0 = c - nth * per, c1 = min(per, c0 + end - c);
        c += c1 - c0;
        const int e = __builtin_amdgcn_readfirstlane(l.active[nth]), count = __builtin_amdgcn_readfirstlane(l.count[e]), first = __builtin_amdgcn_readfirstlane(l.start[e]);
        const float alpha = B == 16 ? a.down.tensor_scales[e] * kUnit : kUnit;
        const uint8_t *wc[NT], *ws[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t at = (int64_t)e * a.down.rows + min(n0 + 16 * t + i, a.N - 1);
            wc[t] = a.down.codes + at * a.down.code_pitch;
            ws[t] = a.down.scales + at * a.down.scale_pitch;
        }
        auto tokens = [&](auto mt_tag, int r0) {
            constexpr int MT = decltype(mt_tag)::value;
            const uint16_t* row[MT];
            bool valid[MT];
#pragma unroll
            for (int r = 0; r < MT; ++r) {
                const int which = r0 + 8 * r + (i & 7);
                valid[r] = which < count;
                row[r] = (i < 8 ? a.high : a.low) + (int64_t)l.slots[first + min(which, count - 1)] * a.I;
            }
            float4v acc[1][MT][NT];
            clear<MT, NT>(acc);
            accumulate<B, MT, NT>(row, valid, wc, ws, a.I, c0, c1, acc);
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int which = r0 + 8 * r + 4 * (q & 1) + k;
                    float* to = own + l.slots[first + min(which, count - 1)] / a.top * COLS + i;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        // lanes of the first half hold sums of high numbers, those of the second of low ones of the same rows
                        const uint2v both = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[0][r][t][k]), __float_as_uint(acc[0][r][t][k]), false, false);
                        const float v = __builtin_fmaf(__uint_as_float(both[1]), kLow, __uint_as_float(both[0]));
                        if (lane < 32 && which < count) to[16 * t] += v * alpha;
                    }
                }
        };
        for (int r0 = 0; r0 < count; r0 += 32) {
            if (count - r0 <= 8) tokens(std::integral_constant<int, 1>{}, r0);
            else if (count - r0 <= 16) tokens(std::integral_constant<int, 2>{}, r0);
            else tokens(std::integral_constant<int, 4>{}, r0);
        }
    }
    __syncthreads();
    for (int idx = tid; idx < a.M * COLS; idx += THREADS) {
        const int m = idx / COLS, n = n0 + idx % COLS;
        if (n >= a.N) continue;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += sums[w * a.M * COLS + idx];
        if (a.residual) sum += (float)a.residual[m * a.ldr + n];
        store_out(a.y + m * a.ldy + n, sum);
    }
}

// Bytes of a launch's parts of the workspace.
struct MoeWorkspace {
    size_t reordered, half;                     // rows in the weights' order; one of the two numbers of h
};
MoeWorkspace workspace_of(int64_t M, int64_t top, int64_t K, int64_t I, bool reorder) {
    auto whole = [](int64_t bytes) { return ((size_t)bytes + 255) / 256 * 256; };
    return {reorder ? whole(M * K * 2) : 0, whole(M * top * I * 2)};
}

template <int B, typename OutT>
arcq_status launch_tokens(const MoeArgs& p, int64_t m0, int64_t M) {
    const MoeWorkspace w = workspace_of(std::min<int64_t>(p.M, kMostTokens), p.top, p.K, p.I, p.perm != nullptr);
    uint8_t* at = static_cast<uint8_t*>(p.workspace);
    uint16_t *reordered = reinterpret_cast<uint16_t*>(at), *high = reinterpret_cast<uint16_t*>(at + w.reordered), *low = reinterpret_cast<uint16_t*>(at + w.reordered + w.half);
    const uint16_t* x = static_cast<const uint16_t*>(p.x) + m0 * p.ldx;
    int64_t ldx = p.ldx;
    if (p.perm) {
        if (arcq_status st = launch_reorder_rows(x, M, p.K, p.ldx, p.perm, reordered, p.stream)) return st;
        x = reordered, ldx = p.K;
    }
    const int32_t* ids = p.ids + m0 * p.top;
    const int64_t most = std::min<int64_t>(p.E, M * p.top);            // experts that there can be work for
    const int tiles = (int)(p.I / 16);
    const Experts up = {p.up_codes, p.up_scales, p.up_tensor_scales, (p.K + p.S_up) / 2, (p.K + p.S_up) / B, (int)(2 * p.I)};
    const Experts down = {p.down_codes, p.down_scales, p.down_tensor_scales, (p.I + p.S_down) / 2, (p.I + p.S_down) / B, (int)p.N};
    const UpArgs u = {x, ldx, ids, p.weights + m0 * p.top, (int)M, (int)p.top, (int)p.E, (int)p.K, (int)p.I, p.activation, up, high, low, tiles};
    hipLaunchKernelGGL((up_kernel<B, 8>), dim3((unsigned)(most * tiles)), dim3(512), 0, p.stream, u);
    if (arcq_status st = check_launch("up_kernel")) return st;
    const DownArgs<OutT> d = {high, low, ids, (int)M, (int)p.top, (int)p.E, (int)p.I, (int)p.N, down, static_cast<const OutT*>(p.residual) + (p.residual ? m0 * p.ldr : 0), p.ldr,
                              static_cast<OutT*>(p.y) + m0 * p.ldy, p.ldy};
    constexpr int NT = 1, WAVES = 8;
    auto kern = down_kernel<B, NT, WAVES, OutT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3((unsigned)((p.N + 16 * NT - 1) / (16 * NT))), dim3(64 * WAVES), sizeof(Lists) + (size_t)(WAVES * M * 16 * NT * 4), p.stream, d);
    return check_launch("down_kernel");
}

}  // namespace

size_t moe_workspace_bytes(int64_t M, int64_t top, int64_t K, int64_t I, bool reorder) {
    const MoeWorkspace w = workspace_of(std::min<int64_t>(M, kMostTokens), top, K, I, reorder);
    return w.reordered + 2 * w.half;
}

// Tokens go kMostTokens at a time.
arcq_status launch_moe(int block, const MoeArgs& p) {
    for (int64_t m = 0; m < p.M; m += kMostTokens) {
        const int64_t rows = std::min<int64_t>(p.M - m, kMostTokens);
        const arcq_status st = block == 16 ? (p.y_dtype == ARCQ_DTYPE_F16 ? launch_tokens<16, _Float16>(p, m, rows) : launch_tokens<16, float>(p, m, rows))
                                           : (p.y_dtype == ARCQ_DTYPE_F16 ? launch_tokens<32, _Float16>(p, m, rows) : launch_tokens<32, float>(p, m, rows));
        if (st) return st;
    }
    return ARCQ_OK;
}

}  // namespace arcq
