// MXFP8 activations times packed MXFP4 weights: y[m,n] = sum_b 2^(sa[m,b]-127) 2^(sw[n,b]-127) sum_{i<32} a[m,32b+i] qw[n,32b+i],
// b over the K / 32 primary blocks, a E4M3, qw E2M1, fp32 accumulation.
//
// gfx950 multiplies the two formats natively: v_mfma_scale_f32_{16x16x128,32x32x64}_f8f6f4 takes a format per operand and one E8M0 scale per
// 32 k and row of each; with an 8-bit operand it runs at half of its FP4 rate.
// With an 8-bit operand the unit lines up the eight products of eight consecutive k at the largest of them and drops what lies more than 13 bits
// below its exponent (measured one product at a time; sums of such groups, and the accumulator, keep 24 bits).  E4M3 x E2M1 products span
// 22 bits, so with outlier channels a product of 512 k was 2.7e-5 off (norm of the error over that of the result, fp32 accumulation: 5e-8).
// SPLIT multiplies twice, once with the elements of 2 and more (bit 6 of the code) and once with the others, zeros in their places: products
// of the first kind lie between 2^-3 and 2^11, those of the second between 2^-10 and 2^4, nothing is dropped, and fp32 accumulation is
// the only rounding.
// What a lane supplies (checked on the GPU with one element at a time), lane (i, q) of 16 or 32 rows and 4 or 2 groups:
//   4-bit operand  k = 32 q .. 32 q + 31                                   16 bytes: one block
//   8-bit operand  k = 16 q .. 16 q + 15 and half of the step's k further  32 bytes: half of one block, half of another
//   scale          of block q of the step, for either operand
#include "gemm_decode.h"
#include "gemm_epilogue.h"
#include "internal.h"

#include <algorithm>
#include <type_traits>

namespace arcq {

namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

// The codes with bit 6, and those without, zeros in the others' places.
__device__ __forceinline__ void split_codes(const int8v& a, int8v& large, int8v& small) {
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        const uint32_t v = (uint32_t)a[w], bit = v & 0x40404040u;
        const uint32_t l = v & ((bit << 2) - (bit >> 6));       // 0xFF for every byte that has the bit
        large[w] = (int)l;
        small[w] = (int)(v ^ l);
    }
}

// Weight-streaming kernel: tiles of 16 MT rows by 16 NT weight rows, K split over the WAVES waves of a workgroup.  Bound by reading the
// weights once (17/32 byte per weight) for a few rows; any sizes.
template <int MT, int NT, int WAVES, typename OutT>
__global__ __launch_bounds__(WAVES * 64) void mx8_stream_kernel(
    const uint8_t* __restrict__ a_codes, const uint8_t* __restrict__ a_scales, const uint8_t* __restrict__ w_codes,
    const uint8_t* __restrict__ w_scales, int M, int N, int nb, int nbw, OutT* __restrict__ y, int64_t ldy, uint32_t tiles_n) {
    __shared__ float red[WAVES][MT * NT][4][64];
    static_assert(sizeof(red) <= 64 * 1024, "partial tiles must fit the static LDS limit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int i = lane & 15, q = lane >> 4;
    const int n0 = (int)(blockIdx.x % tiles_n) * (16 * NT), m0 = (int)(blockIdx.x / tiles_n) * (16 * MT);
    const uint8_t *ac[MT], *as[MT], *wc[NT], *ws[NT];
#pragma unroll
    for (int r = 0; r < MT; ++r) {
        const int m = min(m0 + 16 * r + i, M - 1);                  // rows past M repeat row M-1 and are not stored
        ac[r] = a_codes + (int64_t)m * nb * 32;
        as[r] = a_scales + (int64_t)m * nb;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int n = min(n0 + 16 * t + i, N - 1);
        wc[t] = w_codes + (int64_t)n * nbw * 16;
        ws[t] = w_scales + (int64_t)n * nbw;
    }
    float4v acc[MT][NT];
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = float4v{0.f, 0.f, 0.f, 0.f};

    const int chunks = (nb + 3) >> 2;               // of 128 k; the last one may hold fewer than four blocks
    for (int c = wave; c < chunks; c += WAVES) {
        const int b = min(4 * c + q, nb - 1);       // blocks past the end: the last one's bytes, and weight codes of zero
        const bool ok = 4 * c + q < nb;
        const int a0 = min(128 * c + 16 * q, 32 * nb - 16), a1 = min(128 * c + 64 + 16 * q, 32 * nb - 16);
        uint4 lo[MT], hi[MT], cw[NT];
        uint32_t sa[MT], sw[NT];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            lo[r] = *reinterpret_cast<const uint4*>(ac[r] + a0);
            hi[r] = *reinterpret_cast<const uint4*>(ac[r] + a1);
            sa[r] = as[r][b];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            cw[t] = *reinterpret_cast<const uint4*>(wc[t] + 16 * (int64_t)b);
            sw[t] = ws[t][b];
        }
        int8v large[MT], small[MT];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            const int8v a = {(int)lo[r].x, (int)lo[r].y, (int)lo[r].z, (int)lo[r].w, (int)hi[r].x, (int)hi[r].y, (int)hi[r].z, (int)hi[r].w};
            split_codes(a, large[r], small[r]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int8v w = {ok ? (int)cw[t].x : 0, ok ? (int)cw[t].y : 0, ok ? (int)cw[t].z : 0, ok ? (int)cw[t].w : 0, 0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < MT; ++r) {
                // formats 0: E4M3, 4: E2M1
                acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(small[r], w, acc[r][t], 0, 4, 0, (int)sa[r], 0, (int)sw[t]);
                acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(large[r], w, acc[r][t], 0, 4, 0, (int)sa[r], 0, (int)sw[t]);
            }
        }
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
        if (m < M && n < N) store_out(y + (int64_t)m * ldy + n, sum);
    }
}

struct Mx8Args {
    const uint8_t *a_codes, *a_scales, *w_codes, *w_scales;
    int M, N, nb, nbw;
    int64_t ldy;
    hipStream_t stream;
};

template <int MT, int NT, typename OutT>
arcq_status launch_stream(const Mx8Args& a, OutT* y) {
    const unsigned tiles_n = ((unsigned)a.N + 16 * NT - 1) / (16 * NT), tiles_m = ((unsigned)a.M + 16 * MT - 1) / (16 * MT);
    hipLaunchKernelGGL((mx8_stream_kernel<MT, NT, 8, OutT>), dim3(tiles_n * tiles_m), dim3(512), 0, a.stream, a.a_codes, a.a_scales, a.w_codes, a.w_scales, a.M, a.N,
                       a.nb, a.nbw, y, a.ldy, tiles_n);
    return check_launch("mx8_stream_kernel");
}

template <typename OutT>
arcq_status launch_typed(const Mx8Args& a, OutT* y) {
    if (a.M <= 16) return a.N <= 4096 ? launch_stream<1, 1>(a, y) : launch_stream<1, 4>(a, y);
    if (a.M <= 32) return a.N <= 4096 ? launch_stream<2, 1>(a, y) : launch_stream<2, 4>(a, y);
    return launch_stream<4, 2>(a, y);
}

}  // namespace

size_t mx8_gemm_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

arcq_status launch_mx8_gemm(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* w_codes, const uint8_t* w_scales, int64_t M,
                            int64_t N, int64_t K, int64_t S, void* y, int y_dtype, int64_t ldy, void* workspace, hipStream_t stream) {
    (void)workspace;
    const Mx8Args a = {a_codes, a_scales, w_codes, w_scales, (int)M, (int)N, (int)(K >> 5), (int)((K + S) >> 5), ldy, stream};
    return y_dtype == ARCQ_DTYPE_F16 ? launch_typed(a, static_cast<_Float16*>(y)) : launch_typed(a, static_cast<float*>(y));
}

}  // namespace arcq
