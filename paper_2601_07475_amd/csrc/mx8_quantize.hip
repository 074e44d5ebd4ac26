// MXFP8 activations: blocks of 32 E4M3 elements with one E8M0 (power-of-two) scale, in the channel order of the packed weights;
// alone (the input of a projection behind an activation function) or behind the residual's addition and RMSNorm.
//
//   h = fl16(x + residual);  ms = fl32(exact sum of h^2 / K);  rstd = 1 / sqrt(ms + eps);  y = fl16(fl16(fl32(h rstd)) gamma)
//   block of 32: E = floor(log2(max |y|)) - 8, code = E4M3(y 2^-E), round to nearest even, saturating at 448
//
// (The roundings of the norm are those of arcq_rmsnorm_quantize_act.)  Everything but the element's rounding is exact: scaling by a
// power of two.  Bound by memory: 2 bytes in and 1 + 1/32 out per element, with the addition 4 and 3 + 1/32.
//
// A workgroup owns whole rows.  A lane owns 16 consecutive channels at a time (32 bytes in, 16 out), the two lanes of a block are neighbours and
// exchange their maxima by one data-parallel-primitive move.  A row is asked for while the one before it is being processed, in
// registers: the addition, the new hidden state and the sum of squares want it in its own order; only the reordered values go through LDS.
//
// Measured (us, and TB/s of what is read and written, the order apart):    quantize        norm          addition and norm
//        1 x 14336, reordered                                              3.6           4.9               5.4      (2.4 the launch of one row)
//      333 x 5120                                                          2.7  1.9      4.8  1.1          4.8  2.5  (norm alone: reordered)
//     2048 x 8192, reordered                                              10.4  4.9     14.3  3.6         21.4  5.5
//     8192 x 8192, reordered                                              32.2  6.3     41.6  4.9         89    5.3
//     8192 x 28672, reordered                                            136    5.2    178    4.0        356    4.6
// (The last line with inputs that change from pass to pass, 125 to 129 us for the quantizer where they are the same; the others with the same, of
// which the caches have a part.)  Single rows are bound by one compute unit's way to memory and the launch, the others by memory.  From 333 rows on the
// norm takes 29 to 39 % more than the quantizer alone (barriers), the reads of LDS in the order of the weights 4 to 30 % more than none.
#include "internal.h"
#include "lds_dma.h"
#include "row_stats.h"

#include <hip/hip_fp16.h>

namespace arcq {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float pair_max(float a) {
    const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(a), 0xB1, 0xF, 0xF, true);   // quad_perm [1,0,3,2]
    return fmaxf(a, __int_as_float(o));
}

// A lane's half of a block -> 16 codes and the block's scale byte (the same in both lanes of the block).
__device__ __forceinline__ uint4 quantize_half(const float (&v)[16], bool scale_up, uint32_t& sbyte) {
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(v[i]));
    amax = pair_max(amax);
    // amax is zero or a normal fp32 number: its exponent field is floor(log2) + 127
    const uint32_t bits = __float_as_uint(amax);
    sbyte = amax > 0.0f ? (bits >> 23) - 8u + (scale_up && (bits & 0x7FFFFFu) > 0x600000u ? 1u : 0u) : 127u;
    const float inv = __uint_as_float((254u - sbyte) << 23);            // 2^-E, exact
    uint32_t c[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        // the conversion turns what rounds past 448 into NaN: saturate in front of it
        auto q = [&](int e) { return __builtin_amdgcn_fmed3f(v[4 * w + e] * inv, -448.0f, 448.0f); };
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(q(0), q(1), 0, false);
        c[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q(2), q(3), p, true);
    }
    return make_uint4(c[0], c[1], c[2], c[3]);
}

// The channels' wider forms that came before are not kept for what comes behind, at two registers a channel and more.
template <int HPT>
__device__ __forceinline__ void pin(uint32_t (&h)[HPT][8]) {
#pragma unroll
    for (int j = 0; j < HPT; ++j)
#pragma unroll
        for (int w = 0; w < 8; ++w) asm volatile("" : "+v"(h[j][w]));
}

constexpr int kStatWords = 5 * 64;      // 64-bit words behind the row: two rows' partial sums, three exact ones

// HPT     halves (16 channels) a lane owns: 1, 2, or 4 for rows of more than 32768 channels, which are not asked for ahead (registers)
//         (HPT 2 with gamma kept in registers, too, spills: 4096 x 28672 with addition, norm and order 246 us, here 185.  HPT 4 with the norm does
//         so by 36 or 88 bytes a lane, beside the 56 or 112 that it has in and out.)
// ADD     the residual is added in front, and the sum stored as the new hidden state
// NORM    RMSNorm in front of the quantizer: one more barrier, behind which the row in LDS is known to have been read
// GATHER  channels are reordered, through LDS: two buffers without NORM, as far as they fit, so that one barrier a row is enough
// STREAM  inputs far larger than the caches: non-temporal loads
template <int HPT, bool ADD, bool NORM, bool GATHER, bool STREAM>
__global__ __launch_bounds__(1024) void mx8_rows_kernel(
    const uint16_t* x, int64_t ldx, const uint16_t* residual, int64_t ldr, uint16_t* hidden, int64_t ldh, int rows, int K,
    const uint16_t* __restrict__ gamma, float eps, double delta, double inv_K, const int32_t* __restrict__ perm,
    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, uint32_t flags) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr bool AHEAD = HPT <= 2;
    constexpr int BUFFERS = !GATHER ? 0 : NORM || !AHEAD ? 1 : 2;
    const bool scale_up = (flags & ARCQ_SCALE_ROUND_UP) != 0;
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63;
    const int halves = K >> 4;
    const uint32_t row_bytes = 2u * (uint32_t)K;
    double* stats = reinterpret_cast<double*>(lds + (size_t)BUFFERS * row_bytes);

    uint32_t row = blockIdx.x;              // (32 bits of an unsigned number hold the last row and a grid behind it)
    if (row >= (uint32_t)rows) return;

    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    int at[HPT];
    bool live[HPT];                         // (both lanes of a block are, or neither)
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        live[j] = tid + j * T < halves;
        at[j] = live[j] ? tid + j * T : halves - 1;
    }
    auto fetch = [&](const uint16_t* base, int64_t ld, uint32_t r, u32x4 (&to)[HPT][2]) {
#pragma unroll
        for (int j = 0; j < HPT; ++j) {
            const u32x4* src = reinterpret_cast<const u32x4*>(base + (int64_t)r * ld) + 2 * at[j];
#pragma unroll
            for (int p = 0; p < 2; ++p) to[j][p] = STREAM ? __builtin_nontemporal_load(src + p) : src[p];
        }
    };
    u32x4 in[HPT][2], in2[ADD ? HPT : 1][2];
    auto ask = [&](uint32_t r) {
        fetch(x, ldx, r, in);
        if constexpr (ADD) fetch(residual, ldr, r, in2);
    };
    if (AHEAD) ask(row);

    // Source channels and gamma, two to a register: kept, or gamma in LDS (HPT 2), or read again for every row (HPT 4).
    auto channels_of = [&](int j, uint32_t (&to)[8]) {
        const int4* pp = reinterpret_cast<const int4*>(perm + 16 * at[j]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int4 v4 = pp[q];
            to[2 * q] = ((uint32_t)v4.x & 0xFFFFu) | ((uint32_t)v4.y << 16);
            to[2 * q + 1] = ((uint32_t)v4.z & 0xFFFFu) | ((uint32_t)v4.w << 16);
        }
    };
    constexpr bool KEEP_CHAN = GATHER && HPT <= 2, KEEP_GAMMA = NORM && HPT == 1, LDS_GAMMA = NORM && HPT == 2;
    uint32_t chan[KEEP_CHAN ? HPT : 1][8], gam[KEEP_GAMMA ? HPT : 1][8];
    uint4* lds_gamma = reinterpret_cast<uint4*>(lds + (size_t)BUFFERS * row_bytes + (NORM ? 8 * kStatWords : 0));
#pragma unroll
    for (int j = 0; j < HPT; ++j) {
        if constexpr (KEEP_CHAN) channels_of(j, chan[j]);
        if constexpr (KEEP_GAMMA || LDS_GAMMA) {
            const uint4* gp = reinterpret_cast<const uint4*>(gamma + 16 * at[j]);
            const uint4 g0 = gp[0], g1 = gp[1];
            if constexpr (KEEP_GAMMA) {
                gam[j][0] = g0.x, gam[j][1] = g0.y, gam[j][2] = g0.z, gam[j][3] = g0.w;
                gam[j][4] = g1.x, gam[j][5] = g1.y, gam[j][6] = g1.z, gam[j][7] = g1.w;
            } else if (live[j]) {           // read by the lane that stores it
                lds_gamma[2 * at[j]] = g0;
                lds_gamma[2 * at[j] + 1] = g1;
            }
        }
    }
    uint32_t turn = 0;
    for (; row < (uint32_t)rows; row += gridDim.x, turn ^= 1u) {
        if (!AHEAD) ask(row);
        uint32_t h[HPT][8];                 // the lane's channels, two to a register
#pragma unroll
        for (int j = 0; j < HPT; ++j)
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                h[j][w] = in[j][w >> 2][w & 3];
                if constexpr (ADD) {
                    const uint32_t r = in2[j][w >> 2][w & 3];       // (a value: a bit cast of a vector's element in place takes the first one)
                    h[j][w] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, h[j][w]) + __builtin_bit_cast(half2v, r));
                }
            }
        const uint32_t next = row + gridDim.x;
        if (AHEAD && next < (uint32_t)rows) ask(next);
        if constexpr (ADD) {
#pragma unroll
            for (int j = 0; j < HPT; ++j)
                if (live[j]) {
                    uint4* to = reinterpret_cast<uint4*>(hidden + (int64_t)row * ldh) + 2 * at[j];
                    to[0] = make_uint4(h[j][0], h[j][1], h[j][2], h[j][3]);
                    to[1] = make_uint4(h[j][4], h[j][5], h[j][6], h[j][7]);
                }
        }
        if constexpr (NORM) {
            // Mean of squares, defined with an EXACT sum.  A plain fp64 sum S^ of the squares (each exact) passes through fewer than
            // 150 roundings a term, so S^ = S (1 + t), |t| < 150 * 2^-53; with delta = (K + 260) 2^-52 the fp32 roundings of
            // S^ (1 - delta) / K and S^ (1 + delta) / K bracket that of the exactly summed value, because every rounding
            // is monotone.  If the two agree, that is the answer; a row in some 10^5 takes the integer sum below.
            bool decided = false;
            float rstd = 0.0f;
            if (!(flags & ARCQ_RMSNORM_EXACT_SUM)) {
                double part = 0.0;
#pragma unroll
                for (int j = 0; j < HPT; ++j) {
                    double s16 = 0.0;
#pragma unroll
                    for (int w = 0; w < 8; ++w) {
                        const half2v p = __builtin_bit_cast(half2v, h[j][w]);
                        s16 = __builtin_fma((double)p[0], (double)p[0], s16);
                        s16 = __builtin_fma((double)p[1], (double)p[1], s16);
                    }
                    part += live[j] ? s16 : 0.0;
                }
                part = row16_sum(part);
                if ((tid & 15) == 0) stats[64 * turn + (tid >> 4)] = part;
            }
            wait_lgkmcnt0();
            wg_barrier();                   // not __syncthreads(): the next row stays in flight
            if (!(flags & ARCQ_RMSNORM_EXACT_SUM)) {
                // every wave finishes the statistics for itself: same sum, same operations, same result
                double sum = row16_sum(16 * lane < T ? stats[64 * turn + lane] : 0.0);
                auto row_of_16 = [&](int r) {
                    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(sum), 16 * r), __builtin_amdgcn_readlane(__double2loint(sum), 16 * r));
                };
                sum = (row_of_16(0) + row_of_16(1)) + (row_of_16(2) + row_of_16(3));
                const double q = sum * inv_K;
                const float ms_lo = (float)(q * (1.0 - delta)), ms_hi = (float)(q * (1.0 + delta));
                decided = ms_lo == ms_hi;
                rstd = 1.0f / __builtin_sqrtf(ms_lo + eps);             // IEEE square root and division
            }
            pin(h);
            if (__builtin_amdgcn_readfirstlane(decided ? 1 : 0) == 0) {     // the same in every wave of the workgroup
                uint64_t s[3] = {0, 0, 0};
#pragma unroll
                for (int j = 0; j < HPT; ++j)
#pragma unroll
                    for (int w = 0; w < 8; ++w)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint64_t v = (uint64_t)(fabs((double)__builtin_bit_cast(half2v, h[j][w])[e]) * 0x1p24);
                            const uint64_t a = v >> 20, b = v & 0xFFFFFu;
                            if (live[j]) {
                                s[0] += a * a;
                                s[1] += a * b;
                                s[2] += b * b;
                            }
                        }
                uint64_t* exact = reinterpret_cast<uint64_t*>(stats + 128);
#pragma unroll
                for (int c = 0; c < 3; ++c) {
#pragma unroll
                    for (int d = 1; d < 16; d <<= 1) s[c] += __shfl_xor((unsigned long long)s[c], d);
                    if ((tid & 15) == 0) exact[64 * c + (tid >> 4)] = s[c];
                }
                wait_lgkmcnt0();
                wg_barrier();
#pragma unroll
                for (int c = 0; c < 3; ++c) {
                    s[c] = 16 * lane < T ? exact[64 * c + lane] : 0;
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) s[c] += __shfl_xor((unsigned long long)s[c], d);
                }
                const float ms = (float)(join_exact_sums(s[0], s[1], s[2]) / (double)K);
                rstd = 1.0f / __builtin_sqrtf(ms + eps);
                pin(h);
            }
#pragma unroll
            for (int j = 0; j < HPT; ++j) {
                uint32_t g[8];
                if constexpr (KEEP_GAMMA) {
#pragma unroll
                    for (int w = 0; w < 8; ++w) g[w] = gam[j][w];
                } else {
                    const uint4* gp = LDS_GAMMA ? lds_gamma + 2 * at[j] : reinterpret_cast<const uint4*>(gamma + 16 * at[j]);
                    const uint4 g0 = gp[0], g1 = gp[1];
                    g[0] = g0.x, g[1] = g0.y, g[2] = g0.z, g[3] = g0.w, g[4] = g1.x, g[5] = g1.y, g[6] = g1.z, g[7] = g1.w;
                }
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    const half2v p = __builtin_bit_cast(half2v, h[j][w]);
                    float a = (float)p[0] * rstd, b = (float)p[1] * rstd;
                    // pinned between the two roundings: multiply and conversion would be fused into one that rounds once
                    asm("" : "+v"(a));
                    asm("" : "+v"(b));
                    const half2v t = {(_Float16)a, (_Float16)b};
                    h[j][w] = __builtin_bit_cast(uint32_t, t * __builtin_bit_cast(half2v, g[w]));
                }
            }
        }
        if constexpr (KEEP_CHAN && HPT == 2) pin(chan);     // (nor are two addresses for each of their pairs)
        const uint32_t base = BUFFERS == 2 ? turn * row_bytes : 0u;
        if constexpr (GATHER) {
#pragma unroll
            for (int j = 0; j < HPT; ++j)
                if (live[j]) {
                    uint4* to = reinterpret_cast<uint4*>(lds + base) + 2 * at[j];
                    to[0] = make_uint4(h[j][0], h[j][1], h[j][2], h[j][3]);
                    to[1] = make_uint4(h[j][4], h[j][5], h[j][6], h[j][7]);
                }
            wait_lgkmcnt0();
            wg_barrier();
        }
#pragma unroll
        for (int j = 0; j < HPT; ++j) {
            float v[16];
            uint32_t from[8];
            if constexpr (GATHER && !KEEP_CHAN) channels_of(j, from);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (GATHER) {
                    const uint32_t ch = ((KEEP_CHAN ? chan[j] : from)[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
                    v[i] = __half2float(*reinterpret_cast<const __half*>(lds + base + 2u * ch));
                } else {
                    v[i] = (float)__builtin_bit_cast(half2v, h[j][i >> 1])[i & 1];
                }
            }
            uint32_t sbyte;
            const uint4 c = quantize_half(v, scale_up, sbyte);
            if (live[j]) {
                *reinterpret_cast<uint4*>(codes + (int64_t)row * K + 16 * at[j]) = c;
                if ((tid & 1) == 0) scales[(int64_t)row * (K >> 5) + (at[j] >> 1)] = (uint8_t)sbyte;
            }
        }
        if (GATHER && !NORM && BUFFERS == 1) {
            wait_lgkmcnt0();
            wg_barrier();
        }
    }
}

struct RowArgs {
    const uint16_t* x;
    int64_t ldx;
    const uint16_t* residual;
    int64_t ldr;
    uint16_t* hidden;
    int64_t ldh;
    int64_t rows, K;
    const uint16_t* gamma;
    float eps;
    const int32_t* perm;
    uint8_t *codes, *scales;
    uint32_t flags;
    hipStream_t stream;
};

template <int HPT, bool ADD, bool NORM, bool GATHER, bool STREAM>
arcq_status launch_rows(const RowArgs& a) {
    auto kern = mx8_rows_kernel<HPT, ADD, NORM, GATHER, STREAM>;
    const int halves = (int)(a.K >> 4), threads = ((halves + HPT - 1) / HPT + 63) / 64 * 64;
    const int buffers = !GATHER ? 0 : NORM || HPT > 2 ? 1 : 2;
    const size_t lds = (size_t)buffers * 2 * (size_t)a.K + (NORM ? 8 * kStatWords : 0) + (NORM && HPT == 2 ? 2 * (size_t)a.K : 0);
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    // as many workgroups as the chip holds at once, never more than rows
    static thread_local int cached_threads = 0, cached_per_cu = 0;
    static thread_local size_t cached_lds = 0;
    if (cached_threads != threads || cached_lds != lds) {
        int n = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, threads, lds) != hipSuccess || n < 1) {
            (void)hipGetLastError();
            n = 1;
        }
        cached_threads = threads;
        cached_lds = lds;
        cached_per_cu = n;
    }
    int64_t wgs = (int64_t)num_cu() * cached_per_cu;
    if (wgs > a.rows) wgs = a.rows;
    const double delta = (double)(a.K + 260) * 0x1p-52;
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(threads), lds, a.stream, a.x, a.ldx, a.residual, a.ldr, a.hidden, a.ldh, (int)a.rows,
                       (int)a.K, a.gamma, a.eps, delta, 1.0 / (double)a.K, a.perm, a.codes, a.scales, a.flags);
    return check_launch("mx8_rows_kernel");
}

template <int HPT, bool STREAM>
arcq_status launch_variant(const RowArgs& a) {
    if (a.residual) return a.perm ? launch_rows<HPT, true, true, true, STREAM>(a) : launch_rows<HPT, true, true, false, STREAM>(a);
    if (a.gamma) return a.perm ? launch_rows<HPT, false, true, true, STREAM>(a) : launch_rows<HPT, false, true, false, STREAM>(a);
    return a.perm ? launch_rows<HPT, false, false, true, STREAM>(a) : launch_rows<HPT, false, false, false, STREAM>(a);
}

}  // namespace

arcq_status launch_mx8_quantize(const void* x, int64_t ldx, const void* residual, int64_t ldr, void* hidden, int64_t ldh, int64_t rows, int64_t K,
                                const void* gamma, float eps, const int32_t* perm, uint8_t* codes, uint8_t* scales, uint32_t flags, hipStream_t stream) {
    const RowArgs a = {static_cast<const uint16_t*>(x), ldx, static_cast<const uint16_t*>(residual), ldr, static_cast<uint16_t*>(hidden), ldh, rows, K,
                       static_cast<const uint16_t*>(gamma), eps, perm, codes, scales, flags, stream};
    const bool far = (uint64_t)rows * (uint64_t)K * 2 > (192ull << 20);     // beyond what the caches can hold
    if (K <= 16384) return far ? launch_variant<1, true>(a) : launch_variant<1, false>(a);
    if (K <= 32768) return far ? launch_variant<2, true>(a) : launch_variant<2, false>(a);
    return far ? launch_variant<4, true>(a) : launch_variant<4, false>(a);
}

}  // namespace arcq
