// MXFP8 activations times packed MXFP4 weights: y[m,n] = sum_b 2^(sa[m,b]-127) 2^(sw[n,b]-127) sum_{i<32} a[m,32b+i] qw[n,32b+i],
// b over the K / 32 primary blocks, a E4M3, qw E2M1, fp32 accumulation.
//
// gfx950 multiplies the two formats natively: v_mfma_scale_f32_{16x16x128,32x32x64}_f8f6f4 takes a format per operand and one E8M0 scale per
// 32 k and row of each; with an 8-bit operand it runs at half of its FP4 rate.
// With an 8-bit operand the unit lines up the eight products of eight consecutive k at the largest sum of two exponents (E2M1's 0.5 counts as one of
// exponent 0) and drops what lies more than 13 bits below it (measured one product at a time; sums of such groups, and the accumulator, keep
// 24 bits).  E4M3 x E2M1 products span 22 bits: 256 x 0.5 hides seven products of 2^-5.2 beside it altogether, and with outlier channels a product of
// 512 k was 2.7e-5 off (norm of the error over that of the result, fp32 accumulation: 5e-8).
// So everything is multiplied twice, for either type of output, once with the elements of 2 and more (bit 6 of the code) and once with the others,
// zeros in their places: bits of the first kind of products lie from 2^-3 on, under exponents up to 10, those of the second from 2^-10 on, under
// exponents up to 2; nothing is dropped, and fp32 accumulation is the only rounding.  The price is twice the matrix unit's time where that bounds.
// What a lane supplies (checked on the GPU with one element at a time), lane (i, q) of 16 or 32 rows and 4 or 2 groups:
//   4-bit operand  k = 32 q .. 32 q + 31                                   16 bytes: one block
//   8-bit operand  k = 16 q .. 16 q + 15 and half of the step's k further  32 bytes: half of one block, half of another
//   scale          of block q of the step, for either operand
// Measured: 8192 x 8192 over K = 28672 2.4 ms (1.6 PFLOP/s of whole products, 3.2 on the matrix unit; from registers alone, with random codes and
// every compute unit busy, the instruction reaches 3.8 at 1.82 GHz: power), fp32 output 2.67 ms; 777 x 6147 over 4352 48 us, fp32 53 (two passes take 22 on
// the matrix unit); 300 x 4096 over 14336 43 us; streaming: 16 x 14336 over 4096 9.4 us (3.3 TB/s of weights), 1 x 4096 over 4096 4.5, either type.
#include "code_rows.h"
#include "epilogue.h"
#include "gemm_decode.h"
#include "gemm_epilogue.h"
#include "internal.h"
#include "lane_transpose.h"
#include "lds_dma.h"
#include "tile_order.h"

#include <algorithm>
#include <atomic>
#include <type_traits>
#include <utility>

namespace arcq {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

// The codes with bit 6, and those without, zeros in the others' places.
__device__ __forceinline__ void split_word(uint32_t v, int8v& large, int8v& small, int w) {
    const uint32_t bit = v & 0x40404040u, l = v & ((bit << 2) - (bit >> 6));       // 0xFF for every byte that has the bit
    large[w] = (int)l;
    small[w] = (int)(v ^ l);
}
__device__ __forceinline__ void split_codes(const int8v& a, int8v& large, int8v& small) {
#pragma unroll
    for (int w = 0; w < 8; ++w) split_word((uint32_t)a[w], large, small, w);
}

// Weight-streaming kernel: tiles of 16 MT rows by 16 NT weight rows, K split over the WAVES waves of a workgroup.  Bound by reading the
// weights once (17/32 byte per weight) for a few rows; any sizes.  Whole chunks of 128 k go four at a time: every code of the four, and their scale
// bytes, four to a load and transposed across the lane groups, are in flight at once.
template <int MT, int NT, int WAVES, typename OutT, typename Ep>
__global__ __launch_bounds__(WAVES * 64) void mx8_stream_kernel(
    const uint8_t* __restrict__ a_codes, const uint8_t* __restrict__ a_scales, const uint8_t* __restrict__ w_codes,
    const uint8_t* __restrict__ w_scales, int M, int N, int nb, int nbw, OutputOf<OutT, Ep> y, int64_t ldy, uint32_t tiles_n, uint32_t tiles_m, int splits, Ep ep) {
    // the partial tiles of BATCH weight tiles fit the static LDS limit at a time
    constexpr int BATCH = WAVES * MT * NT > 64 ? (NT + 1) / 2 : NT;
    __shared__ float red[WAVES][MT * BATCH][4][64];
    static_assert(sizeof(red) <= 64 * 1024, "partial tiles must fit the static LDS limit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int i = lane & 15, q = lane >> 4;
    const uint32_t strip = blockIdx.x / tiles_n, split = strip / tiles_m;           // one of `splits` runs of K, with fp32 partial results of its own
    const int n0 = (int)(blockIdx.x % tiles_n) * (16 * NT), m0 = (int)(strip % tiles_m) * (16 * MT);
    y += (int64_t)split * M * N;
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
    // one chunk; byte `at` of the scale registers
    auto multiply = [&](const int4v (&lo)[MT], const int4v (&hi)[MT], const uint4 (&cw)[NT], const uint32_t (&sa)[MT], const uint32_t (&sw)[NT], auto at) {
        constexpr int AT = decltype(at)::value;
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            const int8v a = __builtin_shufflevector(lo[r], hi[r], 0, 1, 2, 3, 4, 5, 6, 7);
            int8v large, small;
            split_codes(a, large, small);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int8v w = {(int)cw[t].x, (int)cw[t].y, (int)cw[t].z, (int)cw[t].w, 0, 0, 0, 0};
                // formats 0: E4M3, 4: E2M1
                acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(small, w, acc[r][t], 0, 4, AT, (int)sa[r], AT, (int)sw[t]);
                acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(large, w, acc[r][t], 0, 4, AT, (int)sa[r], AT, (int)sw[t]);
            }
        }
    };

    const int groups = nb >> 4, group0 = (int)split * groups / splits, group1 = ((int)split + 1) * groups / splits;
    const uint32_t sel_half = half_selector(q), sel_byte = byte_selector(q);
    // scale bytes first: they are needed first, and loads retire in order
    auto load = [&](int g, int4v (&lo)[4][MT], int4v (&hi)[4][MT], uint4 (&cw)[4][NT], uint32_t (&sa)[MT], uint32_t (&sw)[NT]) {
#pragma unroll
        for (int r = 0; r < MT; ++r) sa[r] = load4_a1(as[r] + 16 * (int64_t)g + 4 * q);
#pragma unroll
        for (int t = 0; t < NT; ++t) sw[t] = load4_a1(ws[t] + 16 * (int64_t)g + 4 * q);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
#pragma unroll
            for (int t = 0; t < NT; ++t) cw[c][t] = *reinterpret_cast<const uint4*>(wc[t] + 256 * (int64_t)g + 64 * c + 16 * q);
#pragma unroll
            for (int r = 0; r < MT; ++r) {
                lo[c][r] = *reinterpret_cast<const int4v*>(ac[r] + 512 * (int64_t)g + 128 * c + 16 * q);
                hi[c][r] = *reinterpret_cast<const int4v*>(ac[r] + 512 * (int64_t)g + 128 * c + 64 + 16 * q);
            }
        }
        __builtin_amdgcn_sched_barrier(0);      // every load of the group ahead of the first use
    };
    auto compute = [&](const int4v (&lo)[4][MT], const int4v (&hi)[4][MT], const uint4 (&cw)[4][NT], uint32_t (&sa)[MT], uint32_t (&sw)[NT]) {
#pragma unroll
        for (int r = 0; r < MT; ++r) sa[r] = transpose_scale_bytes(sa[r], sel_half, sel_byte);
#pragma unroll
        for (int t = 0; t < NT; ++t) sw[t] = transpose_scale_bytes(sw[t], sel_half, sel_byte);
        multiply(lo[0], hi[0], cw[0], sa, sw, std::integral_constant<int, 0>{});
        multiply(lo[1], hi[1], cw[1], sa, sw, std::integral_constant<int, 1>{});
        multiply(lo[2], hi[2], cw[2], sa, sw, std::integral_constant<int, 2>{});
        multiply(lo[3], hi[3], cw[3], sa, sw, std::integral_constant<int, 3>{});
    };
    for (int g = group0 + wave; g < group1; g += WAVES) {
        int4v lo[4][MT], hi[4][MT];
        uint4 cw[4][NT];
        uint32_t sa[MT], sw[NT];
        load(g, lo, hi, cw, sa, sw);
        compute(lo, hi, cw, sa, sw);
    }
    // what is left, a chunk at a time, in the last run; the last chunk may hold fewer than four blocks
    const int chunks = (int)split + 1 == splits ? (nb + 3) >> 2 : 0;
    for (int c = 4 * groups + (wave - (group1 - group0) % WAVES + WAVES) % WAVES; c < chunks; c += WAVES) {
        const int b = min(4 * c + q, nb - 1);       // blocks past the end: the last one's bytes, and weight codes of zero
        const bool ok = 4 * c + q < nb;
        const int a0 = min(128 * c + 16 * q, 32 * nb - 16), a1 = min(128 * c + 64 + 16 * q, 32 * nb - 16);
        int4v lo[MT], hi[MT];
        uint4 cw[NT];
        uint32_t sa[MT], sw[NT];
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            lo[r] = *reinterpret_cast<const int4v*>(ac[r] + a0);
            hi[r] = *reinterpret_cast<const int4v*>(ac[r] + a1);
            sa[r] = as[r][b];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 v = *reinterpret_cast<const uint4*>(wc[t] + 16 * (int64_t)b);
            cw[t] = make_uint4(ok ? v.x : 0, ok ? v.y : 0, ok ? v.z : 0, ok ? v.w : 0);
            sw[t] = ws[t][b];
        }
        multiply(lo, hi, cw, sa, sw, std::integral_constant<int, 0>{});
    }
#pragma unroll
    for (int t0 = 0; t0 < NT; t0 += BATCH) {
        if (t0 > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int t = t0; t < (t0 + BATCH < NT ? t0 + BATCH : NT); ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) red[wave][r * BATCH + t - t0][e][lane] = acc[r][t][e];
        __syncthreads();
        for (int idx = threadIdx.x; idx < MT * BATCH * 4 * 64; idx += WAVES * 64) {
            const int rt = idx >> 8, e = (idx >> 6) & 3, l = idx & 63;
            if (NT % BATCH != 0 && t0 + rt % BATCH >= NT) continue;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += red[w][rt][e][l];
            const int m = m0 + 16 * (rt / BATCH) + 4 * (l >> 4) + e, n = n0 + 16 * (t0 + rt % BATCH) + (l & 15);
            if (m < M && n < N) store_out(y + (int64_t)m * ldy + n, finish<OutT>(ep, sum, m, n));
        }
    }
}

// Tiled kernel: 32 WM GM by 32 WN GN outputs a workgroup of GM x GN waves, one tile of 32 WM by 32 WN a wave.  A unit is 128 k: per row 128 bytes
// of A and 64 of W.  Units travel global -> LDS with buffer copies through a ring of NS slots, NS - 1 units ahead, one barrier a unit.
// The 16-byte pieces of a row are stored XOR-swizzled, those of A with (row >> 1) & 7, those of W with (row >> 2) & 3, so that 16 consecutive rows, which a
// 16-byte read is served in, lie on 16 different groups of banks; applied by choosing which piece a lane fetches.
// Scale bytes: a row's four of a unit start at any address, copies at dwords.  A window of 16 bytes from the dword on that holds the first byte has
// those of three units whatever the address; readers take two words of it and shift.  Windows have two buffers in front of the ring and are
// asked for three units ahead.  (Through registers instead, the compiler's wait for them was one for every copy in flight.)
// Blocks past the end of a row count as zero weight codes with a scale of 1.
template <int WM, int WN, int GM, int GN, int NS_>
struct Mx8Tile {
    static constexpr int BM = 32 * WM * GM, BN = 32 * WN * GN, NT = 64 * GM * GN, NS = NS_;
    static constexpr int NA = BM * 8 / NT, NW = BN * 4 / NT;                // copies of a unit
    static constexpr int W_CODES = BM * 128, UNIT = W_CODES + BN * 64;
    static constexpr int GROUP = 3;                                         // units of a window
    static constexpr int SCALES = (BM + BN) * 16, UNITS = 2 * SCALES;       // a buffer of windows: rows of A, then of W; where the ring starts
    static constexpr int BLOCKS = (BM + BN) / 64, NSC = (BLOCKS + GM * GN - 1) / (GM * GN);      // copies of 64 windows, and of a wave
    static constexpr int LDS_BYTES = UNITS + NS * UNIT;
    static_assert(BM * 8 % NT == 0 && BN * 4 % NT == 0 && BM % 64 == 0 && BN % 64 == 0, "whole copies");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS of a compute unit");
    static_assert(NS >= 3 && NS - 2 <= GROUP, "windows asked for at the start of a group are older than the copies that its last unit leaves in flight");
    static_assert((NS - 2) * (NA + NW) < 64, "counted wait");
    static_assert(WM * WN >= 2, "half a k-step behind the barrier");
};

__device__ __forceinline__ float16v mfma_w4a8(const uint4& w, const int8v& a, const float16v& c, uint32_t sw, uint32_t sa, int t) {
    const int8v vw = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    // formats 4: E2M1, 0: E4M3; the scale of a lane is byte 2t of its scale register
    return t == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vw, a, c, 4, 0, 0, (int)sw, 0, (int)sa)
                  : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vw, a, c, 4, 0, 2, (int)sw, 2, (int)sa);
}

template <int WM, int WN, int GM, int GN, int NS, typename OutT, typename Ep>
__global__ __launch_bounds__(64 * GM * GN) void mx8_tile_kernel(
    const uint8_t* __restrict__ a_codes, const uint8_t* __restrict__ a_scales, const uint8_t* __restrict__ w_codes,
    const uint8_t* __restrict__ w_scales, int M, int N, int nb, int nbw, OutputOf<OutT, Ep> y, int64_t ldy, int tiles_m, int tiles_n,
    int group_rows, int splits, int64_t split_stride, Ep ep) {
    using C = Mx8Tile<WM, WN, GM, GN, NS>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // With splits > 1 workgroup split * num_tiles + tile adds up a run of K and stores an fp32 partial tile at y + split * split_stride
    const int num_tiles = tiles_m * tiles_n;
    const int split = splits > 1 ? (int)blockIdx.x / num_tiles : 0;
    const TileOrder tile((int)blockIdx.x - split * num_tiles, tiles_m, tiles_n, group_rows);

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r = lane & 31, h = lane >> 5;
    const int wg_m0 = tile.m * C::BM, wg_n0 = tile.n * C::BN;
    const int wrow0 = (wave / GN) * (32 * WM), wcol0 = (wave % GN) * (32 * WN);

    const int nunit = (nb + 3) >> 2;
    int u0 = 0, u1 = nunit;                     // this workgroup's run of units
    if (splits > 1) {
        u0 = (int)((uint32_t)(split * nunit) / (uint32_t)splits);
        u1 = (int)((uint32_t)((split + 1) * nunit) / (uint32_t)splits);
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

    // ---- windows of scale bytes: a wave copies those of 64 rows of one operand at a time (the last copies of some waves repeat others')
    const uint32_t base_a = (uint32_t)(uintptr_t)a_scales & 3u, base_w = (uint32_t)(uintptr_t)w_scales & 3u;
    // (whole words that hold a byte of the operand)
    const buffer_t win_a = buffer_of(a_scales - base_a, (base_a + (uint32_t)M * (uint32_t)nb + 3u) & ~3u);
    const buffer_t win_w = buffer_of(w_scales - base_w, (base_w + (uint32_t)N * (uint32_t)nbw + 3u) & ~3u);
    uint32_t win_row[C::NSC];
#pragma unroll
    for (int e = 0; e < C::NSC; ++e) {
        const int block = min((int)(wave_slot >> 6) + e * GM * GN, C::BLOCKS - 1), row = 64 * block + lane;
        win_row[e] = (64 * block < C::BM ? base_a + (uint32_t)min(wg_m0 + row, M - 1) * (uint32_t)nb
                                         : base_w + (uint32_t)min(wg_n0 + row - C::BM, N - 1) * (uint32_t)nbw) & ~3u;
    }
    auto issue_windows = [&](int group) {       // group of the run
#pragma unroll
        for (int e = 0; e < C::NSC; ++e) {
            const int block = min((int)(wave_slot >> 6) + e * GM * GN, C::BLOCKS - 1);
            const uint32_t to = lds_address(lds) + (group & 1) * C::SCALES + 1024u * (uint32_t)block, from = 4u * (uint32_t)(u0 + C::GROUP * group);
            if (64 * block < C::BM) copy16(win_a, win_row[e], from, to);
            else copy16(win_w, win_row[e], from, to);
        }
    };
    // a lane's bytes of a unit's word of its rows, shifted so that they are bytes 0 and 2 (rows 32 apart have the same place in a word)
    const uint32_t shift_a = 8u * ((base_a + (uint32_t)r * (uint32_t)nb & 3u) + h), shift_w = 8u * ((base_w + (uint32_t)r * (uint32_t)nbw & 3u) + h);

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
    uint32_t sa[WM], sw[WN];
    auto read_a = [&](int t, int i, const uint8_t* st) {
#pragma unroll
        for (int p = 0; p < 2; ++p) fa[t][i][p] = *reinterpret_cast<const uint4*>(st + rd_a + i * 4096 + 16u * ((uint32_t)(4 * t + 2 * p + h) ^ swz_a));
    };
    auto read_w = [&](int t, int j, const uint8_t* st) {
        fw[t][j] = *reinterpret_cast<const uint4*>(st + rd_w + j * 2048 + 16u * ((uint32_t)(2 * t + h) ^ swz_w));
    };
    // part k of `parts` of a k-step's fragments, in the order that the MFMAs want them
    auto read_part = [&](int t, int k, int parts, const uint8_t* st) {
        constexpr int ALL = WM + WN;
#pragma unroll
        for (int f = 0; f < ALL; ++f)
            if (f * parts / ALL == k) {
                if (f == 0) read_a(t, 0, st);
                else if (f <= WN) read_w(t, f - 1, st);
                else read_a(t, f - WN, st);
            }
    };
    uint2 na[WM], nw[WN];
    auto read_scales = [&](int group, int word) {
        const uint8_t* at = lds + (group & 1) * C::SCALES + 4 * word;
        auto two = [&](int row) {
            const uint32_t* v = reinterpret_cast<const uint32_t*>(at + 16 * row);
            return make_uint2(v[0], v[1]);
        };
#pragma unroll
        for (int i = 0; i < WM; ++i) na[i] = two(wrow0 + 32 * i + r);
#pragma unroll
        for (int j = 0; j < WN; ++j) nw[j] = two(C::BM + wcol0 + 32 * j + r);
    };
    auto take_scales = [&]() {
#pragma unroll
        for (int i = 0; i < WM; ++i) sa[i] = (uint32_t)(((uint64_t)na[i].y << 32 | na[i].x) >> shift_a);
#pragma unroll
        for (int j = 0; j < WN; ++j) sw[j] = (uint32_t)(((uint64_t)nw[j].y << 32 | nw[j].x) >> shift_w);
    };

    // ---- a unit, scheduled by hand: 2 WM WN pairs of MFMAs.  Everything else goes between them, behind the first one, so that the
    // matrix unit does not wait for it: the copies of unit u + NS - 1 (its slot was last read in unit u - 1, which every wave left before
    // the barrier inside unit u - 1), the reads of k-step 1's fragments, and, behind the barrier that opens unit u + 1 before the last half
    // k-step, the reads of that unit's first fragments and scale bytes.
    // COPY: there is a unit u + NS - 1.  DRAIN: there is not, but more units follow.  LAST: none does.
    enum { COPY, DRAIN, LAST };
    constexpr int NM = WM * WN, NDMA = C::NA + C::NW, LAST_Q = 2 * NM - NM / 2;
    constexpr int FIRST = NM >= 8 ? 4 : NM >= 4 ? 2 : 1;        // MFMA slots that read the fragments of k-step 1
    constexpr int NEXT = NM >= 16 ? 3 : 1;                      // and, from LAST_Q on, those of the next unit's k-step 0
    constexpr int COPY0 = NM >= 4 ? 1 : 0;                      // first slot with a copy; all are ahead of the wait that counts them
    constexpr int SPREAD = LAST_Q - COPY0;
    int slot = 0, word = 0, group = 0;                          // of unit u
    int8v large[2], small[2];                                   // codes of the fragment being multiplied and of the next
    auto run_unit = [&](int u, auto phase_tag) {
        constexpr int PHASE = decltype(phase_tag)::value;
        const uint8_t* st = lds + C::UNITS + slot * C::UNIT;
        const int slot1 = slot == NS - 1 ? 0 : slot + 1, fill = slot == 0 ? NS - 1 : slot - 1;
        const int word1 = word == C::GROUP - 1 ? 0 : word + 1, group1 = word1 == 0 ? group + 1 : group;
        bool last = false;
        uint32_t va = 0, vw = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if (PHASE == LAST && t == 1 && ragged && 4 * u + 2 >= nb) break;
            if (PHASE == LAST && ragged && 4 * u + 2 * t + h >= nb) {
#pragma unroll
                for (int i = 0; i < WM; ++i) sa[i] = 0x7F7F7F7Fu;
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    fw[t][j] = make_uint4(0, 0, 0, 0);
                    sw[j] = 0x7F7F7F7Fu;
                }
            }
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                constexpr int TURNS = 2 * WM;
                const int turn = t * WM + i;
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    const int q = t * NM + i * WN + j;
                    if (q == LAST_Q && PHASE != LAST) {
                        // unit u + 1 has landed: the copies of later units are younger (and so are no windows that are read below)
                        if constexpr (PHASE == COPY) {
                            wait_vmcnt<(NS - 2) * NDMA>();
                        } else {
                            const int later = u1 - 2 - u;       // units in flight behind u + 1
                            if (NS >= 5 && later == 2) wait_vmcnt<2 * NDMA>();
                            else if (NS >= 4 && later == 1) wait_vmcnt<NDMA>();
                            else wait_vmcnt<0>();
                        }
                        wait_lgkmcnt0();                        // (every fragment of unit u has arrived)
                        wg_barrier();
                    }
                    if (PHASE != LAST && q >= LAST_Q && q < LAST_Q + NEXT) {
                        read_part(0, q - LAST_Q, NEXT, lds + C::UNITS + slot1 * C::UNIT);
                        if (q == LAST_Q + NEXT - 1) read_scales(group1, word1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    // weights as the row operand: see store_tile_swapped
                    acc[i][j] = mfma_w4a8(fw[t][j], small[turn & 1], acc[i][j], sw[j], sa[i], t);
                    acc[i][j] = mfma_w4a8(fw[t][j], large[turn & 1], acc[i][j], sw[j], sa[i], t);
                    __builtin_amdgcn_sched_barrier(0);
                    if (q == 0) {
                        if (PHASE != LAST && word == 0 && u + C::GROUP < u1) issue_windows(group + 1);
                        if constexpr (PHASE == COPY) {
                            last = ragged && u + NS - 1 == nunit - 1;
                            va = lane_a(u + NS - 1, last);
                            vw = lane_w(u + NS - 1, last);
                        }
                    }
                    if (q < FIRST) read_part(1, q, FIRST, st);
                    if (PHASE == COPY && q >= COPY0 && q < LAST_Q) {
#pragma unroll
                        for (int d = 0; d < NDMA; ++d)
                            if (COPY0 + d * SPREAD / NDMA == q) issue_one(d, u + NS - 1, fill, va, vw, last);
                    }
                    // the next fragment's two kinds of codes, behind the second half of this one's MFMAs
                    constexpr int HALF = WN / 2;
                    if (j >= HALF && (turn + 1 < TURNS || PHASE != LAST)) {
                        const int n = (turn + 1) % TURNS;
                        const uint4(&f)[2] = fa[n / WM][n % WM];
#pragma unroll
                        for (int w = 0; w < 8; ++w)
                            if (w * (WN - HALF) / 8 == j - HALF) {
                                const uint4& v = f[w >> 2];
                                split_word((w & 3) == 0 ? v.x : (w & 3) == 1 ? v.y : (w & 3) == 2 ? v.z : v.w, large[(turn + 1) & 1], small[(turn + 1) & 1], w);
                            }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if constexpr (PHASE != LAST) take_scales();
        slot = slot1;
        word = word1;
        group = group1;
    };

    issue_windows(0);
#pragma unroll
    for (int k = 0; k < NS - 1; ++k) {
        const int unit = min(u0 + k, u1 - 1);       // (a run shorter than the ring copies its last unit again)
        const bool last = ragged && unit == nunit - 1;
#pragma unroll
        for (int d = 0; d < NDMA; ++d) issue_one(d, unit, k, lane_a(unit, last), lane_w(unit, last), last);
    }
    wait_vmcnt<(NS - 2) * NDMA>();
    wg_barrier();
    read_part(0, 0, 1, lds + C::UNITS);
    read_scales(0, 0);
    take_scales();
    const uint4 f0 = fa[0][0][0], f1 = fa[0][0][1];
    split_codes(int8v{(int)f0.x, (int)f0.y, (int)f0.z, (int)f0.w, (int)f1.x, (int)f1.y, (int)f1.z, (int)f1.w}, large[0], small[0]);
    int u = u0;
    for (; u < u1 - (NS - 1); ++u) run_unit(u, std::integral_constant<int, COPY>{});
    for (; u < u1 - 1; ++u) run_unit(u, std::integral_constant<int, DRAIN>{});
    run_unit(u, std::integral_constant<int, LAST>{});
    wait_vmcnt<0>();                            // no copy may still be in flight when the LDS is released

    const int m0 = wg_m0 + wrow0, n0 = wg_n0 + wcol0;
    if constexpr (std::is_same<Ep, Epilogue<OutT>>::value) {
        static_assert(epilogue_lds_bytes(WN) * GM * GN <= C::LDS_BYTES, "one epilogue region per wave must fit");
        wg_barrier();                           // every wave has read its last operands: the ring is free
        finish_tile<WM, WN>(acc, lds + wave * epilogue_lds_bytes(WN), m0, n0, lane, M, N, y, ldy, ep);
    } else if constexpr (std::is_same<OutT, _Float16>::value) {
        static_assert(epilogue_lds_bytes(WN) * GM * GN <= C::LDS_BYTES, "one epilogue region per wave must fit");
        wg_barrier();                           // every wave has read its last operands: the ring is free
        uint8_t* region = lds + wave * epilogue_lds_bytes(WN);
        if constexpr (WM == 1) store_fragment_rows_f16_via_lds<WM, WN, 0, 1>(acc, region, m0, n0, lane, M, N, 1.0f, y, ldy);
        else store_tile_f16_via_lds<WM, WN>(acc, region, m0, n0, lane, M, N, 1.0f, y, ldy);
    } else {
        store_tile_swapped<WM, WN>(acc, m0, n0, r, h, M, N, 1.0f, y + (int64_t)split * split_stride, ldy);
    }
}

struct Mx8Args {
    const uint8_t *a_codes, *a_scales, *w_codes, *w_scales;
    int M, N, nb, nbw;
    int64_t ldy;
    hipStream_t stream;
    EpilogueArgs epilogue;
};

// The kernels' last argument: nothing (NoEpilogue), or what a.epilogue says.
template <typename Ep>
Ep epilogue_of(const Mx8Args& a) {
    if constexpr (std::is_same<Ep, NoEpilogue>::value) return Ep{};
    else return Ep{static_cast<const _Float16*>(a.epilogue.bias), static_cast<decltype(Ep::residual)>(a.epilogue.residual), a.epilogue.ldr, a.epilogue.activation};
}

template <int MT, int NT, typename OutT, typename Ep>
arcq_status launch_stream(const Mx8Args& a, OutT* y, int splits, int64_t /* runs of the workspace are M N apart */) {
    const unsigned tiles_n = ((unsigned)a.N + 16 * NT - 1) / (16 * NT), tiles_m = ((unsigned)a.M + 16 * MT - 1) / (16 * MT);
    hipLaunchKernelGGL((mx8_stream_kernel<MT, NT, 8, OutT, Ep>), dim3(tiles_n * tiles_m * (unsigned)splits), dim3(512), 0, a.stream, a.a_codes, a.a_scales, a.w_codes, a.w_scales, a.M, a.N,
                       a.nb, a.nbw, y, a.ldy, tiles_n, tiles_m, splits, epilogue_of<Ep>(a));
    return check_launch("mx8_stream_kernel");
}

template <int WM, int WN, int NS, typename OutT, typename Ep>
arcq_status launch_tiles(const Mx8Args& a, OutT* y, int splits, int64_t split_stride) {
    using C = Mx8Tile<WM, WN, 2, 2, NS>;
    const int tiles_m = (a.M + C::BM - 1) / C::BM, tiles_n = (a.N + C::BN - 1) / C::BN;
    auto kern = mx8_tile_kernel<WM, WN, 2, 2, NS, OutT, Ep>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3(tiles_m * tiles_n * splits), dim3(C::NT), C::LDS_BYTES, a.stream, a.a_codes, a.a_scales, a.w_codes, a.w_scales,
                       a.M, a.N, a.nb, a.nbw, y, a.ldy, tiles_m, tiles_n, tile_group_rows(tiles_m, tiles_n), splits, split_stride, epilogue_of<Ep>(a));
    return check_launch("mx8_tile_kernel");
}

// The tiles that there are, by fragment rows and columns of a wave and slots of the ring, and what a unit and the rest of a tile take (us): with few
// workgroups, and with every compute unit busy, where two smaller ones share one and large ones meet the power limit.  [0]: products with fp16 output,
// [1]: with fp32; either fitted to measured times of products, in one and several runs of K.  Plans and the launches below are made from this list.
struct Tile {
    int wm, wn, ns;
    double unit_few[2], unit_all[2], rest[2];
};
constexpr Tile kTiles[] = {
    {4, 4, 3, {2.56, 0.00}, {2.43, 0.00}, {0.3, 0.0}},      // one run to an fp16 output only: storing fp32, registers go to scratch
    {3, 4, 3, {1.80, 1.96}, {1.82, 2.17}, {1.8, 5.0}},
    {2, 4, 4, {1.56, 1.36}, {1.33, 1.56}, {1.0, 4.0}},
    {3, 2, 4, {1.57, 1.30}, {1.44, 1.45}, {0.7, 3.5}},
    {2, 2, 3, {0.82, 1.00}, {1.05, 0.81}, {0.4, 2.5}},
    {1, 4, 5, {0.79, 0.95}, {0.77, 0.89}, {1.2, 2.0}},
    {1, 2, 4, {0.54, 0.56}, {0.50, 0.46}, {0.7, 1.5}},
};
constexpr int kTileCount = (int)(sizeof(kTiles) / sizeof(kTiles[0]));
constexpr int first_tile(bool fp32) { return fp32 ? 1 : 0; }
// Most weight tiles a wave of the streaming kernel, with one and with two tiles of 16 rows.
constexpr int kStreamTiles[2] = {7, 4};

struct Mx8Plan {
    int tile = -1, splits = 1;                  // of kTiles, or the streaming kernel with 16 mt rows by 16 nt weight rows
    int mt = 0, nt = 0;
};

// As few weight tiles a wave as keep the launch at one workgroup per compute unit.
Mx8Plan stream_plan(int64_t M, int64_t N) {
    const int64_t tiles = (N + 15) / 16;
    Mx8Plan p;
    p.mt = M <= 16 ? 1 : 2;
    p.nt = (int)std::min<int64_t>((tiles + 255) / 256, kStreamTiles[p.mt - 1]);
    return p;
}

// A function of the sizes, the output's type and whether there is a workspace: whatever a model of their times, fitted to measurements over 32 to 8192
// rows, N = 328 .. 27648 and K = 512 .. 28672, puts first (fp16 output: 1.02x the fastest tile of all on average, 1.3x at worst, over K = 544, of 85
// problems in one run of K, and 1.01x, 1.1x at worst, of 26 in any number; 1 x 512 over 128 streamed 2.5 us, on a tile 3.3).
// The streaming kernel's: 23 ns per load instruction of 16 rows x 64 bytes that a wave issues, of 512 k 4 nt + 8 mt and the scale bytes'; in several
// runs of K where its tiles leave compute units idle (1 x 481 over K = 16032 13.2 -> 5.9 us, 15 x 112 over 20640 14.3 -> 6.7).  With more than 128 rows it
// has what the tiles cannot address.
Mx8Plan plan_mx8(int64_t M, int64_t N, int64_t nb, int64_t nbw, bool fp32, bool workspace) {
    const bool offsets_fit = (uint64_t)M * nb * 32 < 0xFFFF0000ull && (uint64_t)N * nbw * 16 < 0xFFFF0000ull;
    const Mx8Plan stream = stream_plan(M, N);
    if (!offsets_fit) return stream;
    const int64_t units = (nb + 3) >> 2;
    Mx8Plan best;
    double least = 0.0;
    if (M <= 128) {
        const int64_t wgs = ((N + 16 * stream.nt - 1) / (16 * stream.nt)) * ((M + 16 * stream.mt - 1) / (16 * stream.mt));
        for (const int sp : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (sp > 1 && (!workspace || wgs * sp > 256 || nb < 32 * sp)) break;        // runs of at least 1024 k; split only where compute units are idle
            double us = 4.0 + (double)((wgs * sp + 255) / 256) * ((double)nb / (16.0 * sp)) * (double)(5 * stream.nt + 9 * stream.mt) * 0.023;
            if (sp > 1) us = 1.05 * (us + 3.5 + 0.25 * sp + (double)sp * (double)M * (double)N * 8.0 / 4.0e6);
            if (least == 0.0 || us < least) {
                least = us;
                best = stream;
                best.splits = sp;
            }
        }
    }
    for (int i = first_tile(fp32); i < kTileCount; ++i) {
        const Tile& t = kTiles[i];
        const int64_t tiles = ((M + 64 * t.wm - 1) / (64 * t.wm)) * ((N + 64 * t.wn - 1) / (64 * t.wn));
        if (tiles > 0x7FFFFFFF / 8) continue;
        // runs of at least four units, partial results of at most 64 MiB; split only where tiles leave compute units idle
        const int64_t most = workspace && tiles <= 256 && i >= first_tile(true) ? std::min<int64_t>({8, units / 4, (16ll << 20) / (M * N)}) : 1;
        for (int64_t sp = 1; sp == 1 || sp <= most; ++sp) {
            const int64_t work = tiles * sp;
            const double unit = work >= 256 ? t.unit_all[fp32] : t.unit_few[fp32];
            double us = 3.0 + (double)((work + 255) / 256) * ((double)((units + sp - 1) / sp) * unit + t.rest[fp32]);
            if (sp > 1) us += (fp32 ? 3.5 : 2.8) + (double)sp * (double)M * (double)N * 8.0 / 4.0e6;      // fp32 partial results, written and read
            if (least == 0.0 || us < least) {
                least = us;
                best = {i, (int)sp};
            }
        }
    }
    return best;
}

// The launch that a plan names, with an output of OutT.
template <typename OutT>
using Launch = arcq_status (*)(const Mx8Args& a, OutT* y, int splits, int64_t split_stride);

template <typename OutT, typename Ep, size_t... I>
Launch<OutT> tile_launch(int tile, std::index_sequence<I...>) {
    constexpr int FIRST = first_tile(std::is_same<OutT, float>::value);
    static constexpr Launch<OutT> launches[] = {launch_tiles<kTiles[FIRST + I].wm, kTiles[FIRST + I].wn, kTiles[FIRST + I].ns, OutT, Ep>...};
    return launches[tile - FIRST];
}

template <int MT, typename OutT, typename Ep, size_t... I>
Launch<OutT> stream_launch(int nt, std::index_sequence<I...>) {
    static constexpr Launch<OutT> launches[] = {launch_stream<MT, 1 + (int)I, OutT, Ep>...};
    return launches[nt - 1];
}

template <typename OutT, typename Ep>
Launch<OutT> launch_of(const Mx8Plan& p) {
    if (p.tile >= 0) return tile_launch<OutT, Ep>(p.tile, std::make_index_sequence<kTileCount - first_tile(std::is_same<OutT, float>::value)>{});
    return p.mt == 1 ? stream_launch<1, OutT, Ep>(p.nt, std::make_index_sequence<kStreamTiles[0]>{})
                     : stream_launch<2, OutT, Ep>(p.nt, std::make_index_sequence<kStreamTiles[1]>{});
}

// One run of K to y, or several to `partial`, and what adds them up.
template <typename OutT>
arcq_status launch_typed(const Mx8Args& a, OutT* y, float* partial) {
    constexpr bool HALF = std::is_same<OutT, _Float16>::value;
    const Mx8Plan plan = plan_mx8(a.M, a.N, a.nb, a.nbw, !HALF, partial != nullptr);
    const bool more = a.epilogue.any();
    if (plan.splits == 1) return more ? launch_of<OutT, Epilogue<OutT>>(plan)(a, y, 1, 0) : launch_of<OutT, NoEpilogue>(plan)(a, y, 1, 0);
    Mx8Args run = a;
    run.ldy = a.N;
    if (arcq_status st = launch_of<float, NoEpilogue>(plan)(run, partial, plan.splits, (int64_t)a.M * a.N)) return st;
    constexpr int TYPE = HALF ? ARCQ_DTYPE_F16 : ARCQ_DTYPE_F32;
    return more ? launch_splitk_epilogue(partial, plan.splits, a.M, a.N, 1.0f, y, TYPE, a.ldy, a.epilogue, a.stream)
                : launch_splitk_reduce(partial, plan.splits, a.M, a.N, 1.0f, y, TYPE, a.ldy, a.stream);
}

}  // namespace

// Rows of a launch: so many that the tiles can address them (4 GiB of codes) and a grid of the smallest tiles stays within 2^32 threads, for any M.
static int64_t rows_of_launch(int64_t N, int64_t K) {
    const int64_t rows = std::min({0xFFFF0000ll / K, (1ll << 32) / std::max<int64_t>(N, 1), 1ll << 16}) & ~31ll;
    return std::max<int64_t>(rows, 32);
}

size_t mx8_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    M = std::min(M, rows_of_launch(N, K));
    const int one = plan_mx8(M, N, K >> 5, K >> 5, false, true).splits, two = plan_mx8(M, N, K >> 5, K >> 5, true, true).splits;
    const int most = std::max(one, two);
    return most > 1 ? (size_t)most * (size_t)M * (size_t)N * sizeof(float) : 0;
}

void mx8_gemm_route(int64_t M, int64_t N, int64_t K, int64_t S, bool fp32, bool workspace, arcq_route* route) {
    M = std::max<int64_t>(M, 1), N = std::max<int64_t>(N, 1);       // (nothing is launched without rows or features; plans are of some)
    const Mx8Plan p = plan_mx8(std::min(M, rows_of_launch(N, K)), N, K >> 5, (K + S) >> 5, fp32, workspace);
    *route = p.tile >= 0 ? arcq_route{ARCQ_ROUTE_TILES, 64 * kTiles[p.tile].wm, 64 * kTiles[p.tile].wn, p.splits, 0} : arcq_route{ARCQ_ROUTE_STREAM, 16 * p.mt, 16 * p.nt, p.splits, 0};
}

arcq_status launch_mx8_gemm(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* w_codes, const uint8_t* w_scales, int64_t M,
                            int64_t N, int64_t K, int64_t S, void* y, int y_dtype, int64_t ldy, void* workspace, const EpilogueArgs& epilogue,
                            hipStream_t stream) {
    float* partial = static_cast<float*>(workspace);
    const int64_t most = rows_of_launch(N, K);
    for (int64_t m = 0; m < M; m += most) {
        Mx8Args a = {a_codes + m * K, a_scales + m * (K >> 5), w_codes, w_scales, (int)std::min(M - m, most), (int)N, (int)(K >> 5),
                     (int)((K + S) >> 5), ldy, stream, epilogue};
        if (epilogue.residual) a.epilogue.residual = static_cast<const uint8_t*>(epilogue.residual) + m * epilogue.ldr * (y_dtype == ARCQ_DTYPE_F16 ? 2 : 4);
        // (a last run of fewer rows may have a plan of its own, with more runs of K than the workspace was made for: without them)
        float* room = m == 0 || M - m >= most ? partial : nullptr;
        const arcq_status st = y_dtype == ARCQ_DTYPE_F16 ? launch_typed(a, static_cast<_Float16*>(y) + m * ldy, room)
                                                         : launch_typed(a, static_cast<float*>(y) + m * ldy, room);
        if (st) return st;
    }
    return ARCQ_OK;
}

}  // namespace arcq
