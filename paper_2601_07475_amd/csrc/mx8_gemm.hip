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
#include "code_rows.h"
#include "gemm_decode.h"
#include "gemm_epilogue.h"
#include "internal.h"
#include "lds_dma.h"
#include "tile_order.h"

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

// Tiled kernel: 32 WM GM by 32 WN GN outputs a workgroup of GM x GN waves, one tile of 32 WM by 32 WN a wave.  A unit is 128 k: per row 128 bytes
// of A and 64 of W.  Units travel global -> LDS with buffer copies through a ring of three slots, two units ahead, one barrier a unit.
// The 16-byte pieces of a row are stored XOR-swizzled, those of A with (row >> 1) & 7, those of W with (row >> 2) & 3, so that 16 consecutive rows, which a
// 16-byte read is served in, lie on 16 different groups of banks; applied by choosing which piece a lane fetches.
// Scale bytes come for four units at a time, 16 bytes a row, through registers into two buffers in front of the ring: their rows start at any
// address.  Blocks past the end of a row count as zero weight codes.
template <int WM, int WN, int GM, int GN>
struct Mx8Tile {
    static constexpr int BM = 32 * WM * GM, BN = 32 * WN * GN, NT = 64 * GM * GN;
    static constexpr int NA = BM * 8 / NT, NW = BN * 4 / NT;                // copies of a unit
    static constexpr int W_CODES = BM * 128, UNIT = W_CODES + BN * 64;
    static constexpr int SCALES = (BM + BN) * 16, UNITS = 2 * SCALES;       // a buffer of scale bytes: rows of A, then of W; where the ring starts
    static constexpr int LDS_BYTES = UNITS + 3 * UNIT;
    static_assert(BM * 8 % NT == 0 && BN * 4 % NT == 0, "whole copies");
    static_assert(BM <= NT && BN <= NT, "a thread fetches the scale bytes of one row of either operand");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
};

typedef u32x4 u32x4_a1 __attribute__((aligned(1)));
// Scale bytes 16 g .. 16 g + 15 of a row of nb, zeros past its end.
__device__ __forceinline__ uint4 scales_of_units(const uint8_t* row, int nb, int g) {
    const int at = 16 * g;
    if (at + 16 <= nb) {
        const u32x4 v = *reinterpret_cast<const u32x4_a1*>(row + at);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    uint64_t lo = 0, hi = 0;
    if (nb >= 16) {
        const u32x4 v = *reinterpret_cast<const u32x4_a1*>(row + nb - 16);
        lo = (uint64_t)v[1] << 32 | v[0];
        hi = (uint64_t)v[3] << 32 | v[2];
        const int shift = 8 * (at + 16 - nb);       // 8 .. 120
        if (shift >= 64) {
            lo = hi >> (shift - 64);
            hi = 0;
        } else {
            lo = lo >> shift | hi << (64 - shift);
            hi >>= shift;
        }
    } else {
        for (int i = 0; i < nb; ++i) {
            if (i < 8) lo |= (uint64_t)row[i] << (8 * i);
            else hi |= (uint64_t)row[i] << (8 * (i - 8));
        }
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

__device__ __forceinline__ float16v mfma_w4a8(const uint4& w, const int8v& a, const float16v& c, uint32_t sw, uint32_t sa, int t) {
    const int8v vw = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    // formats 4: E2M1, 0: E4M3; the scale of a lane is byte 2t of its scale register
    return t == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vw, a, c, 4, 0, 0, (int)sw, 0, (int)sa)
                  : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vw, a, c, 4, 0, 2, (int)sw, 2, (int)sa);
}

template <int WM, int WN, int GM, int GN, bool SPLIT, typename OutT>
__global__ __launch_bounds__(64 * GM * GN) void mx8_tile_kernel(
    const uint8_t* __restrict__ a_codes, const uint8_t* __restrict__ a_scales, const uint8_t* __restrict__ w_codes,
    const uint8_t* __restrict__ w_scales, int M, int N, int nb, int nbw, OutT* __restrict__ y, int64_t ldy, int tiles_m, int tiles_n,
    int group_rows, int splits, int64_t split_stride) {
    using C = Mx8Tile<WM, WN, GM, GN>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // With splits > 1 workgroup split * num_tiles + tile adds up a run of K and stores an fp32 partial tile at y + split * split_stride
    const int num_tiles = tiles_m * tiles_n;
    const int split = splits > 1 ? (int)blockIdx.x / num_tiles : 0;
    const TileOrder tile((int)blockIdx.x - split * num_tiles, tiles_m, tiles_n, group_rows);

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = lane & 31, h = lane >> 5;
    const int wg_m0 = tile.m * C::BM, wg_n0 = tile.n * C::BN;
    const int wrow0 = (wave / GN) * (32 * WM), wcol0 = (wave % GN) * (32 * WN);

    // this workgroup's run of units [u0, u1), whole groups of four but for the last
    const int nunit = (nb + 3) >> 2;
    int u0 = 0, u1 = nunit;
    if (splits > 1) {
        const int groups = (nunit + 3) >> 2;
        u0 = 4 * (int)((uint32_t)(split * groups) / (uint32_t)splits);
        u1 = min(4 * (int)((uint32_t)((split + 1) * groups) / (uint32_t)splits), nunit);
    }
    const bool ragged = (nb & 3) != 0;

    // ---- copies: eight lanes a row of A, four a row of W
    const uint32_t apitch = (uint32_t)nb * 32u, wpitch = (uint32_t)nbw * 16u;
    const uint32_t pa = (uint32_t)((tid & 7) ^ ((tid >> 4) & 7)), pw = (uint32_t)((tid & 3) ^ ((tid >> 4) & 3));     // piece this lane fetches
    const uint32_t row_a = (uint32_t)(tid >> 3) * apitch, row_w = (uint32_t)(tid >> 2) * wpitch;
    const uint32_t wave_slot = __builtin_amdgcn_readfirstlane((uint32_t)(tid & ~63));
    const uint32_t ring = lds_address(lds) + C::UNITS;
    const CodeRows<C::NT / 8> rows_a(a_codes, M, wg_m0, apitch);
    const CodeRows<C::NT / 4> rows_w(w_codes, N, wg_n0, wpitch);
    auto issue_one = [&](int d, int unit, int slot, uint32_t va, uint32_t vw, bool last) {
        const uint32_t base = ring + slot * C::UNIT + 16u * wave_slot;
        if (d < C::NA) rows_a.issue(d, va, last ? 0u : (uint32_t)unit * 128u, base + 16 * d * C::NT);
        else rows_w.issue(d - C::NA, vw, last ? 0u : (uint32_t)unit * 64u, base + C::W_CODES + 16 * (d - C::NA) * C::NT);
    };
    // in a ragged last unit, pieces past the end repeat the last one
    auto lane_a = [&](int unit, bool last) { return row_a + 16u * (last ? min(8u * unit + pa, 2u * nb - 1u) : pa); };
    auto lane_w = [&](int unit, bool last) { return row_w + 16u * (last ? min(4u * unit + pw, (uint32_t)nb - 1u) : pw); };

    // ---- scale bytes of four units: a row of A and one of W per thread
    const uint8_t* sa_row = a_scales + (int64_t)min(wg_m0 + min(tid, C::BM - 1), M - 1) * nb;
    const uint8_t* sw_row = w_scales + (int64_t)min(wg_n0 + min(tid, C::BN - 1), N - 1) * nbw;
    uint4 next_sa, next_sw;
    auto fetch_scales = [&](int g) {
        next_sa = scales_of_units(sa_row, nb, g);
        next_sw = scales_of_units(sw_row, nb, g);
    };
    auto put_scales = [&](int g) {
        uint8_t* to = lds + (g & 1) * C::SCALES;
        if (C::BM == C::NT || tid < C::BM) *reinterpret_cast<uint4*>(to + 16 * tid) = next_sa;
        if (C::BN == C::NT || tid < C::BN) *reinterpret_cast<uint4*>(to + 16 * (C::BM + tid)) = next_sw;
    };

    // ---- fragments: k-step t of a unit takes pieces 4t + h and 4t + 2 + h of a row of A, piece 2t + h of one of W
    const uint32_t rd_a = (wrow0 + r) * 128, rd_w = C::W_CODES + (wcol0 + r) * 64;
    const uint32_t swz_a = (uint32_t)(r >> 1) & 7u, swz_w = (uint32_t)(r >> 2) & 3u;
    float16v acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    uint4 fa[2][WM][2], fw[2][WN];
    uint32_t sa[WM], sw[WN], sa_n[WM], sw_n[WN];        // shifted so that bytes 0 and 2 are this lane's
    auto read_codes = [&](int t, const uint8_t* st) {
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p) fa[t][i][p] = *reinterpret_cast<const uint4*>(st + rd_a + i * 4096 + 16u * ((uint32_t)(4 * t + 2 * p + h) ^ swz_a));
#pragma unroll
        for (int j = 0; j < WN; ++j) fw[t][j] = *reinterpret_cast<const uint4*>(st + rd_w + j * 2048 + 16u * ((uint32_t)(2 * t + h) ^ swz_w));
    };
    auto read_scales = [&](int unit, uint32_t (&da)[WM], uint32_t (&dw)[WN]) {
        const uint8_t* at = lds + (unit >> 2 & 1) * C::SCALES + 4 * (unit & 3);
#pragma unroll
        for (int i = 0; i < WM; ++i) da[i] = *reinterpret_cast<const uint32_t*>(at + 16 * (wrow0 + 32 * i + r)) >> (8 * h);
#pragma unroll
        for (int j = 0; j < WN; ++j) dw[j] = *reinterpret_cast<const uint32_t*>(at + 16 * (C::BM + wcol0 + 32 * j + r)) >> (8 * h);
    };

    // ---- a unit, scheduled by hand: 2 WM WN MFMAs, or twice as many.  The copies of unit u + 2 go out between the first of them (its slot was last
    // read in unit u - 1, which every wave left before the barrier inside unit u - 1), the fragments of k-step 1 are read while k-step 0 is computed,
    // and the barrier that opens unit u + 1 and the reads of its first fragments come before the last half k-step.
    // LEFT: units behind this one, up to 2.
    constexpr int NM = WM * WN, NDMA = C::NA + C::NW, LAST_Q = 2 * NM - NM / 2;
    static_assert(NDMA <= LAST_Q, "copies are issued ahead of the wait that counts them");
    int slot = 0;
    auto run_unit = [&](int u, auto left_tag) {
        constexpr int LEFT = decltype(left_tag)::value;
        const uint8_t* st = lds + C::UNITS + slot * C::UNIT;
        const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;
        const bool last = ragged && u + 2 == nunit - 1;
        const uint32_t va = lane_a(u + 2, last), vw = lane_w(u + 2, last);
        // scale bytes of the next four units: asked for in the third unit, stored in the fourth, ahead of that unit's copies each
        // (the compiler waits for every copy in flight before it stores them: they are a unit old there)
        const int g1 = (u >> 2) + 1;
        const bool more = LEFT == 2 && 4 * g1 < u1 && (u & 3) == 2, store = LEFT > 0 && 4 * g1 < u1 && (u & 3) == 3;
        if (more) fetch_scales(g1);
        if (store) put_scales(g1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (LEFT == 0 && t == 1 && ragged && 4 * u + 2 >= nb) break;
            if (t == 0) {
                read_codes(1, st);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (LEFT == 0 && ragged && 4 * u + 2 * t + h >= nb) {
#pragma unroll
                for (int j = 0; j < WN; ++j) fw[t][j] = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                const int8v a = {(int)fa[t][i][0].x, (int)fa[t][i][0].y, (int)fa[t][i][0].z, (int)fa[t][i][0].w,
                                 (int)fa[t][i][1].x, (int)fa[t][i][1].y, (int)fa[t][i][1].z, (int)fa[t][i][1].w};
                int8v large, small;
                if constexpr (SPLIT) split_codes(a, large, small);
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    const int q = t * NM + i * WN + j;
                    if (q == LAST_Q && LEFT > 0) {
                        wait_vmcnt<LEFT == 2 ? NDMA : 0>();     // unit u + 1 has landed: the copies of unit u + 2 are younger
                        wait_lgkmcnt0();                        // this wave's scale bytes are stored
                        wg_barrier();
                        read_codes(0, lds + C::UNITS + slot1 * C::UNIT);
                        read_scales(u + 1, sa_n, sw_n);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    // weights as the row operand: see store_tile_swapped
                    if constexpr (SPLIT) {
                        acc[i][j] = mfma_w4a8(fw[t][j], small, acc[i][j], sw[j], sa[i], t);
                        acc[i][j] = mfma_w4a8(fw[t][j], large, acc[i][j], sw[j], sa[i], t);
                    } else {
                        acc[i][j] = mfma_w4a8(fw[t][j], a, acc[i][j], sw[j], sa[i], t);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (LEFT == 2 && q < NDMA) {
                        issue_one(q, u + 2, slot2, va, vw, last);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        if constexpr (LEFT > 0) {
#pragma unroll
            for (int i = 0; i < WM; ++i) sa[i] = sa_n[i];
#pragma unroll
            for (int j = 0; j < WN; ++j) sw[j] = sw_n[j];
        }
        slot = slot1;
    };

    fetch_scales(u0 >> 2);
    put_scales(u0 >> 2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int unit = min(u0 + k, nunit - 1);
        const bool last = ragged && unit == nunit - 1;
#pragma unroll
        for (int d = 0; d < NDMA; ++d) issue_one(d, unit, k, lane_a(unit, last), lane_w(unit, last), last);
    }
    wait_vmcnt<NDMA>();
    wait_lgkmcnt0();
    wg_barrier();
    read_codes(0, lds + C::UNITS);
    read_scales(u0, sa, sw);
    using Left0 = std::integral_constant<int, 0>;
    using Left1 = std::integral_constant<int, 1>;
    using Left2 = std::integral_constant<int, 2>;
    int u = u0;
    for (; u < u1 - 2; ++u) run_unit(u, Left2{});
    if (u1 - u0 > 1) run_unit(u1 - 2, Left1{});
    run_unit(u1 - 1, Left0{});
    wait_vmcnt<0>();                            // no copy may still be in flight when the LDS is released

    const int m0 = wg_m0 + wrow0, n0 = wg_n0 + wcol0;
    if constexpr (std::is_same<OutT, _Float16>::value) {
        static_assert(epilogue_lds_bytes(WN) * GM * GN <= C::LDS_BYTES, "one epilogue region per wave must fit");
        wg_barrier();                           // every wave has read its last operands: the ring is free
        store_tile_f16_via_lds<WM, WN>(acc, lds + wave * epilogue_lds_bytes(WN), m0, n0, lane, M, N, 1.0f, y, ldy);
    } else {
        store_tile_swapped<WM, WN>(acc, m0, n0, r, h, M, N, 1.0f, y + (int64_t)split * split_stride, ldy);
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

template <int WM, int WN, bool SPLIT, typename OutT>
arcq_status launch_tiles(const Mx8Args& a, OutT* y, int splits, int64_t split_stride) {
    using C = Mx8Tile<WM, WN, 2, 2>;
    const int tiles_m = (a.M + C::BM - 1) / C::BM, tiles_n = (a.N + C::BN - 1) / C::BN;
    auto kern = mx8_tile_kernel<WM, WN, 2, 2, SPLIT, OutT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3(tiles_m * tiles_n * splits), dim3(C::NT), C::LDS_BYTES, a.stream, a.a_codes, a.a_scales, a.w_codes, a.w_scales,
                       a.M, a.N, a.nb, a.nbw, y, a.ldy, tiles_m, tiles_n, tile_group_rows(tiles_m, tiles_n), splits, split_stride);
    return check_launch("mx8_tile_kernel");
}

template <typename OutT>
arcq_status launch_typed(const Mx8Args& a, OutT* y) {
    constexpr bool SPLIT = !std::is_same<OutT, _Float16>::value;
    const bool offsets_fit = (uint64_t)a.M * a.nb * 32 < 0xFFFF0000ull && (uint64_t)a.N * a.nbw * 16 < 0xFFFF0000ull;
    if (a.M > 64 && offsets_fit) {
        if ((int64_t)((a.M + 255) / 256) * ((a.N + 255) / 256) >= 192) return launch_tiles<4, 4, SPLIT>(a, y, 1, 0);
        return launch_tiles<2, 2, SPLIT>(a, y, 1, 0);
    }
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
