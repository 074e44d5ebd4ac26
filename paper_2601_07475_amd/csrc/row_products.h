// One chunk of 128 k of a few fp16 rows times packed 4-bit weights on v_mfma_f32_16x16x32_f16, shared by the kernels that do without quantizing the rows.
#pragma once
#include "gemm_decode.h"
#include "lane_transpose.h"

namespace arcq {

typedef float float4v __attribute__((ext_vector_type(4)));
// Eight codes -> fp16, unscaled.
__device__ __forceinline__ half8 widen8(uint32_t c) {
    const half2v p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 1),
                 p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 3);
    return half8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
// E8M0 byte -> 2^(byte - 127); byte 0 is a subnormal.
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte != 0 ? byte << 23 : 0x400000u); }

// Scale bytes of a group of four chunks: lane group q loads chunk q's; every lane gets those it needs of all four, one for each word: all
// bytes of a chunk (MXFP4), or those of its half of the words' blocks of 32 k (NVFP4: even ones for q < 2, odd ones for the others).
__device__ __forceinline__ void spread(uint32_t lower, uint32_t upper, uint32_t (&out)[4]) {
    const uint2v a = __builtin_amdgcn_permlane32_swap(lower, upper, false, false);      // of lane groups q & 1 and (q & 1) + 2
    const uint2v x = __builtin_amdgcn_permlane16_swap(a[0], a[0], false, false), y = __builtin_amdgcn_permlane16_swap(a[1], a[1], false, false);
    out[0] = x[0], out[1] = x[1], out[2] = y[0], out[3] = y[1];
}
template <int B>
__device__ __forceinline__ void scales_of_group(uint2 s, uint32_t (&out)[4]) {
    if constexpr (B == 32) spread(s.x, s.x, out);
    else spread(__builtin_amdgcn_perm(s.y, s.x, 0x06040200u), __builtin_amdgcn_perm(s.y, s.x, 0x07050301u), out);
}

// One chunk of MT row tiles and NT weight tiles.  NVFP4: words 0 and 2, 1 and 3 have accumulators of their own (CH = 2) where a single chain of dependent products
// would make every one wait for the one before.
template <int B, int MT, int NT, int CH>
__device__ __forceinline__ void multiply_chunk(const half8 (&xf)[MT][4], uint4 (&cw)[NT], const uint32_t (&sw)[NT], float4v (&acc)[CH][MT][NT]) {
    half8 w[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        transpose_words(cw[t]);
        const uint32_t word[4] = {cw[t].x, cw[t].y, cw[t].z, cw[t].w};
        const uint32_t s01 = B == 16 ? scale_halves(sw[t], 0x0C010C00) : 0u, s23 = B == 16 ? scale_halves(sw[t], 0x0C030C02) : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][j] = B == 16 ? decode8_half(word[j], j < 2 ? s01 : s23, j & 1) : widen8(word[j]);
    }
    if constexpr (B == 16) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < MT; ++r)
                    acc[j % CH][r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w[t][j], acc[j % CH][r][t], 0, 0, 0);
    } else {
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float4v sum[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w[t][j], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s = power_of(sw[t] >> (8 * j) & 0xFFu);     // of weight row lane % 16, the column that the lane holds sums of
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[0][r][t][e] = __builtin_fmaf(sum[j][e], s, acc[0][r][t][e]);
                }
            }
    }
}

// The same sums kFolded<B> times as large, with every scale in the weights' fp16 numbers.  MXFP4: code x 2^(byte - 127 + 8) is exact in fp16 for bytes from 96 to
// 127, from the smallest subnormal to 1536, which is where weights have theirs: folds() tells whether all of a wave's are.  Chunks with others go block by
// block as above (FOLD: false).  Folding saves 28 of 59 vector instructions for 2048 weights and a tile of rows.
template <int B>
constexpr float kFolded = B == 32 ? 256.0f : 1.0f;

template <int B, int N, int NT>
__device__ __forceinline__ bool folds(const uint32_t (&sw)[N][NT]) {
    if constexpr (B == 16) return true;
    uint32_t off = 0;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int t = 0; t < NT; ++t) off |= sw[d][t] ^ 0x60606060u;
    return __ballot((off & 0xE0E0E0E0u) != 0) == 0;
}

// Tiles of rows 0 .. MT - 1.
template <int B, bool FOLD, int MT, int NT, int ROWS>
__device__ __forceinline__ void multiply_folded(const half8 (&xf)[ROWS][4], uint4 (&cw)[NT], const uint32_t (&sw)[NT], float4v (&acc)[ROWS][NT]) {
    static_assert(MT <= ROWS && (FOLD || B == 32), "NVFP4's scales always fold");
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        transpose_words(cw[t]);
        const uint32_t word[4] = {cw[t].x, cw[t].y, cw[t].z, cw[t].w};
        half8 w[4];
        if constexpr (B == 16) {
            const uint32_t s01 = scale_halves(sw[t], 0x0C010C00), s23 = scale_halves(sw[t], 0x0C030C02);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = decode8_half(word[j], j < 2 ? s01 : s23, j & 1);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = FOLD ? __uint_as_float(((sw[t] >> (8 * j) & 0xFFu) + 8u) << 23) : 1.0f;
                const half2v p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word[j], f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word[j], f, 1),
                             p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word[j], f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word[j], f, 3);
                w[j] = half8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
            }
        }
        if constexpr (FOLD) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < MT; ++r) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w[j], acc[r][t], 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float s = power_of(sw[t] >> (8 * j) & 0xFFu);
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    const float4v sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf[r][j], w[j], float4v{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][t][e] = __builtin_fmaf(sum[e] * kFolded<B>, s, acc[r][t][e]);
                }
            }
        }
    }
}

}  // namespace arcq
