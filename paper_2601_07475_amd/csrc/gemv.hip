// A few fp16 rows times packed 4-bit weights, without quantizing the rows: what a decode step does where the activations stay as they are.
//   y[m,n] = alpha sum_b sw[n,b] sum_{i<B} x[m, perm[B b + i]] qw[n, B b + i],  fp32 accumulation
// over the K primary columns of weights packed as for the 4-bit path (NVFP4: B = 16, E4M3 scales; MXFP4: B = 32, E8M0 scales).
//
// Bound by reading the weights once (9/16 or 17/32 byte per weight).  Codes become fp16 in registers and go to v_mfma_f32_16x16x32_f16 with
// the rows as the 16-row operand, so up to 16 rows cost what one does: 9 to 11 vector instructions per 512 weights, 30 * 10^12 weights a second over
// the chip, twice what 8 TB/s bring.  NVFP4's code x scale product is exact in fp16 (gemm_decode.h).  MXFP4's power of two may leave fp16's
// range: its codes go in as they are, one instruction a block, and the block's sum is scaled in fp32 on its way to the accumulator.
//
// A chunk is 128 k.  Lane (i = lane % 16, q = lane / 16) loads 16 bytes of codes of weight row i (a wave: 16 rows x 64 contiguous bytes) and
// a 4 x 4 transpose of words across the four lane groups (four lane-swap instructions) leaves it with word q of the chunk's blocks of 32 k:
// word j is k = 32 j + 8 q .. + 7, for which the rows' 16 bytes of the four lane groups are contiguous, too.
#include "gemm_decode.h"
#include "gemm_epilogue.h"
#include "internal.h"
#include "lane_transpose.h"

#include <algorithm>
#include <type_traits>

namespace arcq {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));
__device__ __forceinline__ uint4 load16_a1(const uint8_t* p) {
    const u32x4 v = *reinterpret_cast<const u32x4_a1*>(p);
    return uint4{v[0], v[1], v[2], v[3]};
}

// Eight codes -> fp16, unscaled.
__device__ __forceinline__ half8 widen8(uint32_t c) {
    const half2v p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 1),
                 p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 3);
    return half8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
// E8M0 byte -> 2^(byte - 127); byte 0 is a subnormal.
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte != 0 ? byte << 23 : 0x400000u); }

// The scale bytes of a chunk that a lane needs, one for each word: the same for all lane groups (MXFP4), or those of
// its half of the words' blocks of 32 k.
template <int B>
__device__ __forceinline__ uint32_t scales_of_chunk(uint32_t lo, uint32_t hi, uint32_t half_select) {
    return B == 32 ? lo : __builtin_amdgcn_perm(hi, lo, half_select);
}

// One chunk of MT row tiles and NT weight tiles.
template <int B, int MT, int NT>
__device__ __forceinline__ void multiply_chunk(const half8 (&xf)[MT][4], uint4 (&cw)[NT], const uint32_t (&sw)[NT], float4v (&acc)[MT][NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        transpose_words(cw[t]);
        const uint32_t word[4] = {cw[t].x, cw[t].y, cw[t].z, cw[t].w};
        if constexpr (B == 16) {
            const uint32_t s01 = scale_halves(sw[t], 0x0C010C00), s23 = scale_halves(sw[t], 0x0C030C02);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const half8 w = decode8_half(word[j], j < 2 ? s01 : s23, j & 1);
#pragma unroll
                for (int r = 0; r < MT; ++r) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w, acc[r][t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const half8 w = widen8(word[j]);
                const float s = power_of(sw[t] >> (8 * j) & 0xFFu);     // of weight row lane % 16, the column that the lane holds sums of
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    const float4v sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w, float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][t][e] = __builtin_fmaf(sum[e], s, acc[r][t][e]);
                }
            }
        }
    }
}

// B      16: NVFP4, 32: MXFP4
// MT     tiles of 16 rows of x that share every decoded weight;  NT  tiles of 16 weight rows of a workgroup, whose WAVES waves split K
template <int B, int MT, int NT, int WAVES, typename OutT>
__global__ __launch_bounds__(WAVES * 64) void gemv_kernel(
    const uint16_t* __restrict__ x, int64_t ldx, int M, int K, const uint8_t* __restrict__ w_codes, const uint8_t* __restrict__ w_scales,
    int N, int64_t cpitch, int64_t spitch, float alpha, OutT* __restrict__ y, int64_t ldy, uint32_t tiles_n) {
    __shared__ float red[WAVES][MT * NT][4][64];
    static_assert(sizeof(red) <= 64 * 1024, "partial tiles must fit the static LDS limit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int i = lane & 15, q = lane >> 4;
    const int n0 = (int)(blockIdx.x % tiles_n) * (16 * NT), m0 = (int)(blockIdx.x / tiles_n) * (16 * MT);
    constexpr int SB = 128 / B;                     // scale bytes of a chunk
    const uint32_t half_select = q < 2 ? 0x06040200u : 0x07050301u;

    const uint16_t* xr[MT];
#pragma unroll
    for (int r = 0; r < MT; ++r) xr[r] = x + (int64_t)min(m0 + 16 * r + i, M - 1) * ldx;      // rows past M repeat row M-1 and are not stored
    const uint8_t *wc[NT], *ws[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = min(n0 + 16 * t + i, N - 1);
        wc[t] = w_codes + n * cpitch;
        ws[t] = w_scales + n * spitch;
    }
    float4v acc[MT][NT];
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = float4v{0.f, 0.f, 0.f, 0.f};

    // whole chunks, four at a time
    const int groups = K >> 9;
    for (int g = wave; g < groups; g += WAVES) {
        uint4 cw[4][NT], sc[NT][B == 16 ? 2 : 1];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            sc[t][0] = load16_a1(ws[t] + (int64_t)(4 * SB) * g);
            if constexpr (B == 16) sc[t][1] = load16_a1(ws[t] + (int64_t)(4 * SB) * g + 16);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int t = 0; t < NT; ++t) cw[c][t] = load16_a4(wc[t] + 256 * (int64_t)g + 64 * c + 16 * q);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            half8 xf[MT][4];
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[r][j] = *reinterpret_cast<const half8*>(xr[r] + 512 * (int64_t)g + 128 * c + 32 * j + 8 * q);
            uint32_t sw[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (B == 16) {
                    const uint4& s = sc[t][c >> 1];
                    sw[t] = scales_of_chunk<B>(c & 1 ? s.z : s.x, c & 1 ? s.w : s.y, half_select);
                } else {
                    const uint4& s = sc[t][0];
                    sw[t] = c == 0 ? s.x : c == 1 ? s.y : c == 2 ? s.z : s.w;
                }
            }
            multiply_chunk<B, MT, NT>(xf, cw[c], sw, acc);
        }
    }
    // what is left of K, a chunk at a time: blocks past the end count as zero codes, and rows of x are read from their start there
    const int blocks = K / B, chunks = (K + 127) >> 7;
    for (int c = 4 * groups + (wave - groups % WAVES + WAVES) % WAVES; c < chunks; c += WAVES) {
        uint4 cw[NT];
        uint32_t sw[NT];
        const int b0 = B == 16 ? 8 * c + 2 * q : 4 * c + q;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (B == 16) {
                const uint2 lo = load8_a8(wc[t] + 8 * (int64_t)min(b0, blocks - 1)), hi = load8_a8(wc[t] + 8 * (int64_t)min(b0 + 1, blocks - 1));
                const bool ok0 = b0 < blocks, ok1 = b0 + 1 < blocks;
                cw[t] = make_uint4(ok0 ? lo.x : 0, ok0 ? lo.y : 0, ok1 ? hi.x : 0, ok1 ? hi.y : 0);
            } else {
                const uint4 v = load16_a4(wc[t] + 16 * (int64_t)min(b0, blocks - 1));
                const bool ok = b0 < blocks;
                cw[t] = make_uint4(ok ? v.x : 0, ok ? v.y : 0, ok ? v.z : 0, ok ? v.w : 0);
            }
            sw[t] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sw[t] |= (uint32_t)ws[t][min(B == 16 ? 8 * c + 2 * j + (q >> 1) : 4 * c + j, blocks - 1)] << (8 * j);
        }
        half8 xf[MT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 128 * c + 32 * j + 8 * q;
#pragma unroll
            for (int r = 0; r < MT; ++r) xf[r][j] = *reinterpret_cast<const half8*>(xr[r] + (k < K ? k : 0));
        }
        multiply_chunk<B, MT, NT>(xf, cw, sw, acc);
    }
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][r * NT + t][e][lane] = acc[r][t][e];
    __syncthreads();
    for (int idx = threadIdx.x; idx < MT * NT * 4 * 64; idx += WAVES * 64) {
        const int rt = idx >> 8, e = (idx >> 6) & 3, l = idx & 63;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += red[w][rt][e][l];
        const int m = m0 + 16 * (rt / NT) + 4 * (l >> 4) + e, n = n0 + 16 * (rt % NT) + (l & 15);
        if (m < M && n < N) store_out(y + (int64_t)m * ldy + n, sum * alpha);
    }
}

// The rows in the weights' channel order, eight channels a thread, `parts` workgroups a row.
__global__ __launch_bounds__(256) void reorder_rows_kernel(const uint16_t* __restrict__ x, int64_t ldx, int K, const int32_t* __restrict__ perm,
                                                           uint16_t* __restrict__ out, uint32_t parts) {
    const uint32_t m = blockIdx.x / parts;
    const int at = (int)((blockIdx.x - m * parts) * 256 + threadIdx.x) * 8;
    if (at >= K) return;
    const uint16_t* row = x + (int64_t)m * ldx;
    const int4 a = *reinterpret_cast<const int4*>(perm + at), b = *reinterpret_cast<const int4*>(perm + at + 4);
    auto take = [&](int lo, int hi) {       // (an index from an unchecked perm may lie outside the row)
        return (uint32_t)row[min((uint32_t)lo, (uint32_t)K - 1u)] | (uint32_t)row[min((uint32_t)hi, (uint32_t)K - 1u)] << 16;
    };
    *reinterpret_cast<uint4*>(out + (int64_t)m * K + at) = make_uint4(take(a.x, a.y), take(a.z, a.w), take(b.x, b.y), take(b.z, b.w));
}

template <int B, int MT, int NT, typename OutT>
arcq_status launch_tiles(const uint16_t* x, int64_t ldx, int64_t M, int64_t K, const uint8_t* w_codes, const uint8_t* w_scales, int64_t N,
                         int64_t S, float alpha, OutT* y, int64_t ldy, hipStream_t stream) {
    const unsigned tiles_n = (unsigned)((N + 16 * NT - 1) / (16 * NT)), tiles_m = (unsigned)((M + 16 * MT - 1) / (16 * MT));
    hipLaunchKernelGGL((gemv_kernel<B, MT, NT, 8, OutT>), dim3(tiles_n * tiles_m), dim3(512), 0, stream, x, ldx, (int)M, (int)K, w_codes, w_scales,
                       (int)N, (K + S) / 2, (K + S) / B, alpha, y, ldy, tiles_n);
    return check_launch("gemv_kernel");
}

template <int B, typename OutT>
arcq_status launch_typed(const uint16_t* x, int64_t ldx, int64_t M, int64_t K, const uint8_t* w_codes, const uint8_t* w_scales, int64_t N,
                         int64_t S, float alpha, OutT* y, int64_t ldy, hipStream_t stream) {
    const int64_t tiles = (N + 15) / 16;
    const int nt = tiles <= 256 ? 1 : tiles <= 512 || M > 32 ? 2 : 4;
#define ARCQ_GEMV(MT_, NT_) \
    if (nt == NT_) return launch_tiles<B, MT_, NT_>(x, ldx, M, K, w_codes, w_scales, N, S, alpha, y, ldy, stream)
    if (M <= 16) {
        ARCQ_GEMV(1, 1);
        ARCQ_GEMV(1, 2);
        ARCQ_GEMV(1, 4);
    }
    if (M <= 32) {
        ARCQ_GEMV(2, 1);
        ARCQ_GEMV(2, 2);
        ARCQ_GEMV(2, 4);
    }
    ARCQ_GEMV(4, 1);
    return launch_tiles<B, 4, 2>(x, ldx, M, K, w_codes, w_scales, N, S, alpha, y, ldy, stream);
#undef ARCQ_GEMV
}

template <int B>
arcq_status launch_format(const uint16_t* x, int64_t ldx, int64_t M, int64_t K, const uint8_t* w_codes, const uint8_t* w_scales, int64_t N,
                          int64_t S, float alpha, void* y, int y_dtype, int64_t ldy, hipStream_t stream) {
    if (y_dtype == ARCQ_DTYPE_F16)
        return launch_typed<B>(x, ldx, M, K, w_codes, w_scales, N, S, alpha, static_cast<_Float16*>(y), ldy, stream);
    return launch_typed<B>(x, ldx, M, K, w_codes, w_scales, N, S, alpha, static_cast<float*>(y), ldy, stream);
}

}  // namespace

size_t gemv_workspace_bytes(int64_t M, int64_t K, bool reorder) { return reorder ? (size_t)M * (size_t)K * 2 : 0; }

arcq_status launch_gemv(int block, const void* x, int64_t M, int64_t K, int64_t ldx, const int32_t* perm, const uint8_t* w_codes,
                        const uint8_t* w_scales, int64_t N, int64_t S, float alpha, void* y, int y_dtype, int64_t ldy, void* workspace,
                        hipStream_t stream) {
    const uint16_t* rows = static_cast<const uint16_t*>(x);
    if (perm) {
        uint16_t* reordered = static_cast<uint16_t*>(workspace);
        const unsigned parts = (unsigned)((K / 8 + 255) / 256);
        hipLaunchKernelGGL(reorder_rows_kernel, dim3(parts * (unsigned)M), dim3(256), 0, stream, rows, ldx, (int)K, perm, reordered, parts);
        if (arcq_status st = check_launch("reorder_rows_kernel")) return st;
        rows = reordered;
        ldx = K;
    }
    if (block == 16) return launch_format<16>(rows, ldx, M, K, w_codes, w_scales, N, S, alpha, y, y_dtype, ldy, stream);
    return launch_format<32>(rows, ldx, M, K, w_codes, w_scales, N, S, alpha, y, y_dtype, ldy, stream);
}

}  // namespace arcq
