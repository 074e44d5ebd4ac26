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
//
// Loads return in the order they were asked for, so whatever is asked for behind the weights waits for them.  The rows are therefore asked for first
// and reach the matrix instructions through LDS (X):
//   SLICE   a wave brings what it multiplies next, 4 to 16 KB of its own, while it multiplies.  Rows that have to be reordered are so by a launch
//           before, 2.2 to 3 us
//   WHOLE   short rows that have to be reordered: all of them at once, in the order that lanes read them in (a unit of 16 bytes per eight k and
//           row), 0.5 to 1.5 us; one row of 4096 channels over 4096 features 6.1 us where SLICE takes 4.7 without an order
//
// Measured (weights not in cache, rows in order; us, and TB/s of weights):     M = 1         M = 4         M = 16        M = 32
//   NVFP4   4096 features,  4096 channels                                    4.7   2.0     5.0   1.9     6.2   1.5     8.4   1.1
//          27648            5120                                            20.9   3.8    24.6   3.2    29.7   2.7    43.6   1.8
//           8192           28672                                            29.9   4.4    35.8   3.7    42.6   3.1    59.8   2.2
//   MXFP4   4096           14336                                             8.7   3.6     9.3   3.4    13.9   2.2    17.9   1.7
// From 1 to 4 rows the weights' way from memory and the tiles' uneven shares bound it, with more the rows, too: every workgroup reads all of them
// (16 rows: 2 bytes x 16 for every 9 bytes of 16 weights of NT tiles).
#include "gemm_decode.h"
#include "gemm_epilogue.h"
#include "internal.h"
#include "lane_transpose.h"
#include "lds_dma.h"

#include <algorithm>
#include <type_traits>

namespace arcq {

namespace {

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

enum Rows { WHOLE, SLICE };
constexpr int slice_chunks(int rows, int nt, int waves) { return rows == 4 ? 4 : rows == 16 && nt <= 2 && waves == 8 ? 2 : 1; }     // of a wave, as registers allow
constexpr int slice_bytes(int rows, int nt, int waves) { return rows * slice_chunks(rows, nt, waves) * 256; }
constexpr int kWhole = 8192;                    // WHOLE: most values of the rows, 16 a thread

// B      16: NVFP4, 32: MXFP4
// ROWS   most rows of x of a workgroup: 4, 16 or 32, in tiles of 16 that share every decoded weight
// NT     tiles of 16 weight rows of a workgroup, whose WAVES waves split K
// LDS: the rows (WHOLE: M K 2 bytes twice, the second in the channels' own order), then the waves' partial tiles, two sets
template <int B, int ROWS, int NT, int WAVES, int X, typename OutT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(ROWS == 4 || WAVES == 16 ? 4 : 2, 4))) void gemv_kernel(
    const uint16_t* __restrict__ x, int64_t ldx, int M, int K, const int32_t* __restrict__ perm, const uint8_t* __restrict__ w_codes,
    const uint8_t* __restrict__ w_scales, int N, int64_t cpitch, int64_t spitch, float alpha, OutT* __restrict__ y, int64_t ldy, int tiles_n, uint32_t stride, uint32_t splits) {
    constexpr int MT = (ROWS + 15) / 16, THREADS = 64 * WAVES, PIECES = kWhole / 8 / THREADS;
    static_assert(X == SLICE || MT == 1, "WHOLE: up to 16 rows");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = lane & 15, q = lane >> 4;
    // a workgroup takes every stride-th tile of weight rows, for one tile of rows of x
    // and one of `splits` runs of K, with fp32 partial results of its own
    const uint32_t run = blockIdx.x / stride, split = run % splits;
    const int m0 = (int)(run / splits) * ROWS, tile0 = (int)(blockIdx.x % stride);
    y += (int64_t)split * M * N;
    constexpr int SB = 128 / B;                     // scale bytes of a chunk
    const int rows = min(M - m0, ROWS), pieces = K >> 3;

    // Whole chunks of 128 k go to the waves four at a time, in turn, and what is left of them in equal shares.
    const int chunks = K >> 7, chunk0 = (int)(split * (uint32_t)chunks / splits), whole = (int)((split + 1) * (uint32_t)chunks / splits) - chunk0;
    const int rounds = whole / (4 * WAVES), rest = whole - rounds * 4 * WAVES, rest_at = chunk0 + 4 * WAVES * rounds;
    const int rest0 = rest_at + wave * rest / WAVES, rest1 = rest_at + (wave + 1) * rest / WAVES;
    const int turns = rounds + (rest1 > rest0 ? 1 : 0);
    auto first_of = [&](int turn) { return turn < rounds ? chunk0 + 4 * (turn * WAVES + wave) : rest0; };
    auto count_of = [&](int turn) { return turn < rounds ? 4 : turn == rounds ? rest1 - rest0 : 0; };

    // ---- the rows
    u32x4 piece_x[X == WHOLE ? PIECES : 1];
    uint32_t chan[X == WHOLE ? PIECES : 1][4];     // source channels of a piece, two to a register
    if constexpr (X == WHOLE) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int u = tid + p * THREADS;
            if (u < pieces) {
                const int4 a = *reinterpret_cast<const int4*>(perm + 8 * u), b = *reinterpret_cast<const int4*>(perm + 8 * u + 4);
                // (an index from an unchecked perm may lie outside the row)
                auto two = [&](int lo, int hi) { return min((uint32_t)lo, (uint32_t)K - 1u) | min((uint32_t)hi, (uint32_t)K - 1u) << 16; };
                chan[p][0] = two(a.x, a.y), chan[p][1] = two(a.z, a.w), chan[p][2] = two(b.x, b.y), chan[p][3] = two(b.z, b.w);
            }
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int u = tid + p * THREADS;
            if (u < rows * pieces) {
                const int m = rows == 1 ? 0 : u / pieces;
                piece_x[p] = *reinterpret_cast<const u32x4*>(x + (int64_t)(m0 + m) * ldx + 8 * (u - m * pieces));
            }
        }
    }
    // SLICE: piece (eight k) and row at unit ROWS piece + (row ^ swizzle), so that writes of a row and reads of a piece both spread over the
    // banks.  A load instruction brings a row, or two, whole lines of each.
    constexpr int XC = slice_chunks(ROWS, NT, WAVES), LPR = 16 * XC, RPL = 64 / LPR, LOADS = ROWS / RPL;     // chunks of a slice; lanes of a row; rows of a load
    auto unit = [](int piece, int row) { return ROWS * piece + (row ^ (ROWS == 4 ? piece >> 2 & 3 : piece & 15)); };
    uint8_t* slice = lds + (X == SLICE ? wave * slice_bytes(ROWS, NT, WAVES) : 0);
    u32x4 xv[X == SLICE ? LOADS : 1];
    auto load_x = [&](int c) {
        if constexpr (X == SLICE) {
            const int piece = min(16 * c + lane % LPR, pieces - 1);
#pragma unroll
            for (int l = 0; l < LOADS; ++l)
                if (RPL * l < rows) xv[l] = *reinterpret_cast<const u32x4*>(x + (int64_t)min(m0 + RPL * l + lane / LPR, M - 1) * ldx + 8 * piece);
        }
    };
    auto put_x = [&]() {
        if constexpr (X == SLICE) {
#pragma unroll
            for (int l = 0; l < LOADS; ++l)
                if (RPL * l < rows) *reinterpret_cast<u32x4*>(slice + 16 * unit(lane % LPR, RPL * l + lane / LPR)) = xv[l];
        }
    };
    if (turns > 0) load_x(first_of(0));
    __builtin_amdgcn_sched_barrier(0);

    // ---- the weights
    // of the tile whose codes, and of the one whose scales, are asked for
    const uint8_t *wc[NT], *ws[NT];
    auto rows_of = [&](const uint8_t* base, int64_t pitch, int tile, const uint8_t* (&at)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) at[t] = base + min((tile * NT + t) * 16 + i, N - 1) * pitch;
    };
    rows_of(w_codes, cpitch, tile0, wc);
    rows_of(w_scales, spitch, tile0, ws);
    auto load_scales = [&](int c, int count, u32x2 (&sc)[NT]) {      // (past the end: the last chunk's again)
        const int64_t at = (int64_t)SB * (c + min(q, count - 1));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (B == 16) {
                const uint2 v = load8_a1(ws[t] + at);
                sc[t] = u32x2{v.x, v.y};
            } else {
                sc[t] = u32x2{load4_a1(ws[t] + at), 0u};
            }
        }
    };
    auto load_codes = [&](int c, u32x4 (&cw)[NT]) {
#pragma unroll
        for (int t = 0; t < NT; ++t) cw[t] = *reinterpret_cast<const u32x4_a4*>(wc[t] + 64 * (int64_t)c + 16 * q);
    };
    constexpr int AHEAD = MT * NT == 4 ? 2 : 4;          // chunks in flight
    u32x4 cw[AHEAD][NT];
    u32x2 sc[NT];
    if (turns > 0) {
        load_scales(first_of(0), count_of(0), sc);
#pragma unroll
        for (int d = 0; d < AHEAD; ++d)
            if (d < count_of(0)) load_codes(first_of(0) + d, cw[d]);
    }
    __builtin_amdgcn_sched_barrier(0);

    if constexpr (X == WHOLE) {
        uint8_t* to = lds + (size_t)rows * K * 2;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int u = tid + p * THREADS;
            if (u < rows * pieces) *reinterpret_cast<u32x4*>(to + 16 * u) = piece_x[p];
        }
        wait_lgkmcnt0();
        wg_barrier();                               // not __syncthreads(): the weights stay in flight
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int piece = tid + p * THREADS;
            if (piece < pieces)
                for (int m = 0; m < rows; ++m) {
                    auto at = [&](uint32_t ch) { return (uint32_t)*reinterpret_cast<const uint16_t*>(to + 2 * ((uint32_t)m * (uint32_t)K + ch)); };
                    u32x4 v;
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[w] = at(chan[p][w] & 0xFFFFu) | at(chan[p][w] >> 16) << 16;
                    *reinterpret_cast<u32x4*>(lds + 16 * (piece * rows + m)) = v;
                }
        }
        wait_lgkmcnt0();
        wg_barrier();
    }
    // the lane's fragments of chunk c, the d-th of its four
    auto take_x = [&](int c, int d, half8 (&xf)[MT][4]) {
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (X == WHOLE) {
                    xf[r][j] = *reinterpret_cast<const half8*>(lds + 16 * ((16 * c + 4 * j + q) * rows + min(i, rows - 1)));
                } else {
                    xf[r][j] = *reinterpret_cast<const half8*>(slice + 16 * unit(16 * (d % XC) + 4 * j + q, ROWS == 4 ? i & 3 : 16 * r + i));
                }
            }
    };
    constexpr int CH = B == 16 && ROWS == 16 && NT == 1 ? 2 : 1;
    // Partial tiles have two buffers behind the rows, so that a barrier a tile is enough.  The next tile's weights are asked for while this one's are
    // multiplied and added up.
    float* red = reinterpret_cast<float*>(lds + (X == WHOLE ? (uint32_t)rows * (uint32_t)K * 4u : (uint32_t)(WAVES * slice_bytes(ROWS, NT, WAVES))));
    uint32_t turn_red = 0;
    for (int tile = tile0; tile < tiles_n; tile += (int)stride) {
        float4v acc[CH][MT][NT];
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[c][r][t] = float4v{0.f, 0.f, 0.f, 0.f};

        for (int turn = 0; turn < turns; ++turn) {
            const bool over = turn + 1 == turns;
            const int c = first_of(turn), count = count_of(turn);
            const int next = first_of(over ? 0 : turn + 1);
            const int next_count = !over ? count_of(turn + 1) : tile + (int)stride < tiles_n ? count_of(0) : 0;
            const bool next_tile = over && next_count > 0;
            if (next_tile) rows_of(w_scales, spitch, tile + (int)stride, ws);
            uint32_t sw[4][NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                uint32_t s[4];
                scales_of_group<B>(make_uint2(sc[t][0], sc[t][1]), s);
#pragma unroll
                for (int d = 0; d < 4; ++d) sw[d][t] = s[d];
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                if (d < count) {
                    if (d % XC == 0) {
                        put_x();
                        if (d + XC < count) load_x(c + d + XC);
                        else if (next_count > 0) load_x(next);
                    }
                    if (d == 0 && next_count > 0) load_scales(next, next_count, sc);
                    half8 xf[MT][4];
                    take_x(c + d, d, xf);
                    uint4 words[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) words[t] = make_uint4(cw[d % AHEAD][t][0], cw[d % AHEAD][t][1], cw[d % AHEAD][t][2], cw[d % AHEAD][t][3]);
                    multiply_chunk<B, MT, NT, CH>(xf, words, sw[d], acc);
                }
                // AHEAD chunks ahead, as soon as there is room
                if (d + AHEAD == 4 && next_tile) rows_of(w_codes, cpitch, tile + (int)stride, wc);
                if (d + AHEAD < 4) {
                    if (d + AHEAD < count) load_codes(c + d + AHEAD, cw[d % AHEAD]);
                } else if (d + AHEAD - 4 < next_count) {
                    load_codes(next + d + AHEAD - 4, cw[d % AHEAD]);
                }
            }
        }
        // What is left of K, less than a chunk, is for the first wave (the last one has the most): blocks past the end count as zero codes, and rows of x
        // are read from their start there.
        const int blocks = K / B;
        if ((K & 127) != 0 && wave == 0 && split + 1 == splits) {
            int c = chunks;
            asm volatile("" : "+v"(c));             // (its addresses, the same for every tile, are not worth registers in between)
            const uint8_t *tc[NT], *ts[NT];
            rows_of(w_codes, cpitch, tile, tc);
            rows_of(w_scales, spitch, tile, ts);
            uint4 words[NT];
            uint32_t sw[NT];
            const int b0 = B == 16 ? 8 * c + 2 * q : 4 * c + q;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (B == 16) {
                    const uint2 lo = load8_a8(tc[t] + 8 * (int64_t)min(b0, blocks - 1)), hi = load8_a8(tc[t] + 8 * (int64_t)min(b0 + 1, blocks - 1));
                    const bool ok0 = b0 < blocks, ok1 = b0 + 1 < blocks;
                    words[t] = make_uint4(ok0 ? lo.x : 0, ok0 ? lo.y : 0, ok1 ? hi.x : 0, ok1 ? hi.y : 0);
                } else {
                    const uint4 v = load16_a4(tc[t] + 16 * (int64_t)min(b0, blocks - 1));
                    const bool ok = b0 < blocks;
                    words[t] = make_uint4(ok ? v.x : 0, ok ? v.y : 0, ok ? v.z : 0, ok ? v.w : 0);
                }
                sw[t] = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) sw[t] |= (uint32_t)ts[t][min(B == 16 ? 8 * c + 2 * j + (q >> 1) : 4 * c + j, blocks - 1)] << (8 * j);
            }
            half8 xf[MT][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int piece = 16 * c + 4 * j + q, at = piece < pieces ? piece : 0;
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    const int m = min(16 * r + i, rows - 1);            // rows past M repeat the last one and are not stored
                    if constexpr (X == WHOLE) xf[r][j] = *reinterpret_cast<const half8*>(lds + 16 * (at * rows + m));
                    else xf[r][j] = *reinterpret_cast<const half8*>(x + (int64_t)(m0 + m) * ldx + 8 * at);
                }
            }
            multiply_chunk<B, MT, NT, CH>(xf, words, sw, acc);
        }
        float* part = red + turn_red * (WAVES * MT * NT * 256);
        turn_red ^= 1u;
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    part[((wave * MT * NT + r * NT + t) * 4 + e) * 64 + lane] = CH == 2 ? acc[0][r][t][e] + acc[CH - 1][r][t][e] : acc[0][r][t][e];
        wait_lgkmcnt0();
        wg_barrier();                                   // not __syncthreads(): the next tile's weights stay in flight
        for (int idx = tid; idx < MT * NT * 4 * 64; idx += THREADS) {
            const int rt = idx >> 8, e = (idx >> 6) & 3, l = idx & 63;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += part[(w * MT * NT * 4 + rt * 4 + e) * 64 + l];
            const int m = m0 + 16 * (rt / NT) + 4 * (l >> 4) + e, n = (tile * NT + rt % NT) * 16 + (l & 15);
            if (m < min(M, m0 + ROWS) && n < N) store_out(y + (int64_t)m * ldy + n, sum * alpha);
        }
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

struct GemvArgs {
    const uint16_t* x;
    int64_t M, K, ldx;
    const int32_t* perm;
    const uint8_t *w_codes, *w_scales;
    int64_t N, S;
    float alpha;
    int64_t ldy;
    hipStream_t stream;
};

bool whole_rows(int64_t M, int64_t K) { return M <= 4 && M * K <= kWhole; }

struct GemvPlan {
    int nt, splits;
};
// Row tiles that share the decoded weights: 4, 16 or 32 rows, several of the last.
int rows_of(int64_t M) { return M <= 4 ? 4 : M <= 16 ? 16 : 32; }

// The weight tiles of a workgroup (two or four share the rows) and the runs of K, by the least modelled time: a workgroup takes a time in
// proportion to its channels and tiles; K in several runs lets few tiles reach every compute unit and evens out their shares, at the price of
// a launch that adds up partial results.  Measured, us:
//   16 rows, NT = 1, 2, 4: 14336 x 4096 18.6, 13.4, 11.4; 27648 x 5120 43, 35, 30; 8192 x 28672 57, 44, 65; 4096 x 4096 6.8, 8.0, 10.3
//   32 rows, NT = 1, 2:    14336 x 4096 23.7, 17.0; 8192 x 28672 91, 61; 4096 x 4096 8.4, 10.5
//   1, 2, 4, 8 runs:       1 x 1024 x 28672 13.6, 10.5, 8.5, 9.6; 16 x 1024 x 28672 20.6, 14.9, 11.9, 13.9; 30 x 848 x 26208 34.2, 21.6, 14.7, 17.2;
//                          22 x 8490 x 27648 (266 pairs of tiles for 256 compute units) 95, 79, 71; 1 x 4096 x 14336 8.7 in one run, 12 in two
// Against every choice of both on 22 problems the model's was within 6 % of the best but for 1 x 1024 x 14336 and 16 x 1024 x 8192 (15 and 10 %).
GemvPlan plan_gemv(int64_t M, int64_t N, int64_t K, bool reorder) {
    static const double cost[3][3] = {{0.45, 0, 0}, {0.8, 1.4, 2.2}, {1.4, 1.9, 0}};       // us for 1000 channels, NT = 1, 2, 4
    static const int runs[8] = {1, 2, 3, 4, 6, 8, 12, 16};
    const int rows = rows_of(M), r = rows == 4 ? 0 : rows == 16 ? 1 : 2;
    const int64_t tiles_m = (M + rows - 1) / rows;
    const int cus = num_cu();
    GemvPlan best = {1, 1};
    double least = 1e30;
    for (int i = 0; i < 3 && cost[r][i] > 0; ++i) {
        const int nt = 1 << i;
        const int64_t tiles = (N + 16 * nt - 1) / (16 * nt) * tiles_m;
        for (int splits : runs) {
            if (splits > 1 && (splits * 1024 > K || tiles * splits > 8 * cus || (reorder && whole_rows(M, K)))) break;
            const int64_t slots = std::max(cus / splits, 1);
            double us = 2.5 + (double)((tiles + slots - 1) / slots) * cost[r][i] * (double)K / (1000.0 * splits);
            if (splits > 1) us = 1.05 * (us + 3.5 + 0.25 * splits + (double)splits * (double)M * (double)N * 8.0 / 4.0e6);
            if (us < least) least = us, best = {nt, splits};
        }
    }
    return best;
}

template <int B, int ROWS, int NT, int WAVES, int X, typename OutT>
arcq_status launch_tiles(const GemvArgs& a, int splits, OutT* y) {
    auto kern = gemv_kernel<B, ROWS, NT, WAVES, X, OutT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    const size_t rows = X == WHOLE ? (size_t)a.M * a.K * 4 : (size_t)WAVES * slice_bytes(ROWS, NT, WAVES);
    const size_t lds = rows + 2 * (size_t)WAVES * ((ROWS + 15) / 16) * NT * 1024;
    const int64_t tiles_n = (a.N + 16 * NT - 1) / (16 * NT), tiles_m = (a.M + ROWS - 1) / ROWS;
    const int per_cu = ROWS == 4 ? 2 : 1;           // as registers and LDS allow
    const unsigned stride = (unsigned)std::min<int64_t>(tiles_n, std::max(num_cu() * per_cu / splits, 1));
    hipLaunchKernelGGL(kern, dim3(stride * (unsigned)(splits * tiles_m)), dim3(64 * WAVES), lds, a.stream, a.x, a.ldx, (int)a.M, (int)a.K, a.perm,
                       a.w_codes, a.w_scales, (int)a.N, (a.K + a.S) / 2, (a.K + a.S) / B, a.alpha, y, a.ldy, (int)tiles_n, stride, (uint32_t)splits);
    return check_launch("gemv_kernel");
}

// Waves that split K: up to 4 rows, 8, so that two workgroups fit the registers of a compute unit (14336 x 4096 10.8 -> 10.1 us; with 16, 4096 x 4096
// 4.7 -> 5.0).  16 rows, one tile: 16 where each has two chunks of 128 (4096 x 14336 14.9 -> 13.9 us, 1024 x 28672 24.0 -> 20.3; 4096 x 1024 4.3 -> 4.6).
template <int B, typename OutT>
arcq_status launch_planned(const GemvArgs& a, GemvPlan p, OutT* y) {
    if (a.M <= 4) return a.perm ? launch_tiles<B, 4, 1, 8, WHOLE>(a, 1, y) : launch_tiles<B, 4, 1, 8, SLICE>(a, p.splits, y);
    if (a.M <= 16)
        return p.nt == 1   ? (a.K / p.splits >= 4096 ? launch_tiles<B, 16, 1, 16, SLICE>(a, p.splits, y) : launch_tiles<B, 16, 1, 8, SLICE>(a, p.splits, y))
               : p.nt == 2 ? launch_tiles<B, 16, 2, 8, SLICE>(a, p.splits, y)
                           : launch_tiles<B, 16, 4, 8, SLICE>(a, p.splits, y);
    return p.nt == 1 ? launch_tiles<B, 32, 1, 8, SLICE>(a, p.splits, y) : launch_tiles<B, 32, 2, 8, SLICE>(a, p.splits, y);
}

template <int B, typename OutT>
arcq_status launch_typed(const GemvArgs& a, GemvPlan p, OutT* y, float* partial) {
    if (p.splits == 1) return launch_planned<B>(a, p, y);
    GemvArgs run = a;
    run.alpha = 1.0f;
    run.ldy = a.N;
    if (arcq_status st = launch_planned<B>(run, p, partial)) return st;
    return launch_splitk_reduce(partial, p.splits, a.M, a.N, a.alpha, y, std::is_same<OutT, _Float16>::value ? ARCQ_DTYPE_F16 : ARCQ_DTYPE_F32, a.ldy,
                                a.stream);
}

// Rows of a launch: grids and workspaces stay within bounds for any M.
constexpr int64_t kMostRows = 1 << 16;

struct GemvWorkspace {
    size_t reordered, partial;      // bytes of the rows in the weights' order, where no kernel reorders them on the way, and of partial results behind
};
GemvWorkspace gemv_workspace(int64_t M, int64_t N, int64_t K, bool reorder, GemvPlan p) {
    return {reorder && !whole_rows(M, K) ? ((size_t)M * (size_t)K * 2 + 255) / 256 * 256 : 0, p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)N * 4 : 0};
}

template <typename OutT>
arcq_status launch_rows(int block, const GemvArgs& a, GemvPlan p, OutT* y, uint16_t* reordered, float* partial) {
    GemvArgs run = a;
    if (reordered) {
        const unsigned parts = (unsigned)((a.K / 8 + 255) / 256);
        hipLaunchKernelGGL(reorder_rows_kernel, dim3(parts * (unsigned)a.M), dim3(256), 0, a.stream, a.x, a.ldx, (int)a.K, a.perm, reordered, parts);
        if (arcq_status st = check_launch("reorder_rows_kernel")) return st;
        run.x = reordered;
        run.ldx = a.K;
        run.perm = nullptr;
    }
    return block == 16 ? launch_typed<16>(run, p, y, partial) : launch_typed<32>(run, p, y, partial);
}

}  // namespace

size_t gemv_workspace_bytes(int64_t M, int64_t N, int64_t K, bool reorder) {
    const int64_t most = std::min(M, kMostRows);
    const GemvWorkspace w = gemv_workspace(most, N, K, reorder, plan_gemv(most, N, K, reorder));
    return w.reordered + w.partial;
}

arcq_status launch_gemv(int block, const void* x, int64_t M, int64_t K, int64_t ldx, const int32_t* perm, const uint8_t* w_codes,
                        const uint8_t* w_scales, int64_t N, int64_t S, float alpha, void* y, int y_dtype, int64_t ldy, void* workspace,
                        hipStream_t stream) {
    const int64_t most = std::min(M, kMostRows);
    const GemvPlan p = plan_gemv(most, N, K, perm != nullptr);
    const GemvWorkspace w = gemv_workspace(most, N, K, perm != nullptr, p);
    uint16_t* reordered = w.reordered > 0 ? static_cast<uint16_t*>(workspace) : nullptr;
    float* partial = w.partial > 0 ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.reordered) : nullptr;
    for (int64_t m = 0; m < M; m += kMostRows) {
        const int64_t rows = std::min(M - m, kMostRows);
        const GemvArgs a = {static_cast<const uint16_t*>(x) + m * ldx, rows, K, ldx, perm, w_codes, w_scales, N, S, alpha, ldy, stream};
        // (with more rows than a launch takes, the last run goes like the others, in one tile of 32 rows at least: what fits them fits it)
        const arcq_status st = y_dtype == ARCQ_DTYPE_F16 ? launch_rows(block, a, p, static_cast<_Float16*>(y) + m * ldy, reordered, partial)
                                                         : launch_rows(block, a, p, static_cast<float*>(y) + m * ldy, reordered, partial);
        if (st) return st;
    }
    return ARCQ_OK;
}

}  // namespace arcq
