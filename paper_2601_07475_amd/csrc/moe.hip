// The experts of a mixture for a few tokens, on packed 4-bit weights:
//   h[m, j] = w[m, j] act(x[m] G_e^T) (x[m] U_e^T)        e = ids[m, j]            up_few_kernel or up_many_kernel
//   y[m]    = sum_j h[m, j] D_e^T + residual[m]                                    down_few_kernel, or down_many_kernel and join_kernel
// x fp16, G over U the 2 I rows of an expert's first operand, D its second; NVFP4 (B = 16) or MXFP4 (B = 32).
//
// Bound by reading the chosen experts' weights once (3 K I weights each, 9/16 or 17/32 byte a weight).  Tokens are rows of v_mfma_f32_16x16x32_f16's tile, so
// up to 16 (4 behind the activation) cost what one does.  Two launches, because every column of h depends on all of x and every column of y on all of h; what
// a launch that waits for another costs by itself, start, choices and the first trip to memory, is 5 to 6 us, and with few bytes that is most of the time.
//
// Every workgroup finds out by itself which tokens choose an expert: no kernel in front, and none that waits for the host.  An expert that a token
// names twice counts once, with both weights: a token is then in a list once, and sums do not depend on the order of a list.
//
// h goes through memory in fp32.  The second product takes it as two fp16 numbers, what rounds to fp16 and what that leaves, in a unit that goes by the largest value of
// its row, or of its row so far: 23 bits of h, and 2^-38 of that largest value at least, whatever size the values are.  (One fp16 number would put its rounding,
// 2^-12, behind an fp32 y; a fixed unit loses small values and has a largest one.)  Units are powers of two, and sums are taken back exactly.  The two numbers are rows i and
// i + 8 of one row tile, so the second costs no more matrix instructions than the tile's free rows; the halves of a wave hold the sums of either and are put together
// when a wave is done with an expert.
//
// No atomics on results, and every sum in an order that the sizes and choices fix: the same inputs give the same bits.
//
// Measured: us of a call whose inputs and weights change from call to call, TB/s of the chosen experts' weights (a plain read reaches 6.2); and the durations that a trace of
// calls with the same inputs gives of the products' kernels, which overlap at their ends and find part of their weights in caches: they do not add up to the call.
//   one token, eight of 64, 2048 x 1024, MXFP4              17.8   1.5     8.8    9.6
//   one token, two of eight, 4096 x 14336, NVFP4            50.6   3.9    24     19
//   four tokens, eight of 128, 4096 x 1792, MXFP4           86     3.4    49     38
//   13 tokens, four of 30, 5120 x 1392, NVFP4, fp32 y       88 to 98      54     36, reordering and joining 3 to 5 each
//   64 tokens, two of eight, 4096 x 14336, MXFP4           208     3.6   118    114, joining 5
#include "epilogue.h"
#include "internal.h"
#include "lds_dma.h"
#include "row_products.h"

#include <algorithm>
#include <type_traits>

namespace arcq {

namespace {

constexpr int kMostExperts = ARCQ_MOE_MAX_EXPERTS, kMostTokens = 64, kMostSlots = kMostTokens * ARCQ_MOE_MAX_TOP_K;     // of a launch

struct Experts {
    const uint8_t *codes, *scales;              // [E, rows, pitch]
    const float* tensor_scales;                 // NVFP4: [E]
    int64_t code_pitch, scale_pitch;            // bytes of a row
    int rows;                                   // of an expert
};

struct UpArgs {
    const uint16_t* x;
    int64_t ldx;
    const int32_t* ids;
    const float* weights;
    int M, top, E, K, I, activation;
    Experts up;
    float* h;                                   // [M top, pitch]
    int pitch;                                  // I in whole chunks, zeros behind
    uint8_t* exponents;                         // of the largest magnitude of every 16 of a row, [M top, exponents_pitch(tiles)], zeros behind; or null
    int tiles;                                  // of 16 columns
    const int32_t* perm;                        // of up_few_kernel: the order that x is taken in, or null
};

template <typename OutT>
struct DownArgs {
    const float* h;
    const uint8_t* exponents;
    const int32_t* ids;
    int M, top, E, I, pitch, N;
    Experts down;
    const OutT* residual;
    int64_t ldr;
    OutT* y;
    int64_t ldy;
    float* partial;                             // [splits][M top, N]
    int groups, splits;
};

__host__ __device__ constexpr int exponents_pitch(int tiles) { return (tiles + 15) / 16 * 16; }

// The largest over a row of 16 lanes, in all of them.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));        // its neighbour, the pair beside it, the other four, the other eight
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
}

// h of one slot and column; the 16 lanes of a row have the columns of a tile.
__device__ __forceinline__ void store_h(const UpArgs& a, int slot, int n, float g, float u, float weight) {
    float v[1] = {g};
    activate(v, a.activation);
    const float h = v[0] * u * weight;
    float* to = a.h + ((int64_t)slot * a.pitch + n);
    *to = h;
    const bool last = n >= a.I - 16;
    if (last)                                   // whoever has the last tile clears what is left of the last chunk
        for (int z = 16; n + z < a.pitch; z += 16) to[z] = 0.0f;
    if (a.exponents) {
        const uint32_t most = row_max(__float_as_uint(h) & 0x7FFFFFFFu) >> 23;
        uint8_t* row = a.exponents + slot * exponents_pitch(a.tiles);
        const int tile = n >> 4, lane = n & 15;
        if (lane == 0) row[tile] = (uint8_t)most;
        if (last && tile + 1 + lane < exponents_pitch(a.tiles)) row[tile + 1 + lane] = 0;
    }
}

// Values of h below 2^(most - 126) are multiplied by 2^(140 - most) = scale_to(most): the largest lie from 2^13 to 2^14, and those of infinity's neighbours, for which
// `most` is at its end, below 2^16: all are numbers of fp16.  Sums are taken back by scale_from(most).  With kLeast what the two numbers leave is less than fp32 resolves.
constexpr uint32_t kLeast = 14, kMost = 253;
__device__ __forceinline__ float scale_to(uint32_t most) { return __uint_as_float((267u - most) << 23); }
__device__ __forceinline__ float scale_from(uint32_t most) { return __uint_as_float((most - 13u) << 23); }

// The largest magnitude of four values (or something that is not a number).
__device__ __forceinline__ float magnitude(const u32x4& v) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_fabsf(__uint_as_float(v[0])), __builtin_fabsf(__uint_as_float(v[1]))),
                                                                       __builtin_fabsf(__uint_as_float(v[2]))), __builtin_fabsf(__uint_as_float(v[3])));
}
// The largest over the 32 lanes of either half of a wave, in all of them.
__device__ __forceinline__ uint32_t half_wave_max(uint32_t v) {
    v = row_max(v);
    const uint2v rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max(rows[0], rows[1]);
}
// The largest of 16 bytes.
__device__ __forceinline__ uint32_t largest_byte(const u32x4& v) {
    typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
    ushort2v m = {0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, v[k] & 0x00FF00FFu));
        m = __builtin_elementwise_max(m, __builtin_bit_cast(ushort2v, v[k] >> 8 & 0x00FF00FFu));
    }
    return max((uint32_t)m[0], (uint32_t)m[1]);
}
// Four values times scale as fp16 numbers, to `high`, and as fp16 numbers what that leaves, to `low`.
__device__ __forceinline__ void put_h(const u32x4& v, float scale, uint8_t* high, uint8_t* low) {
    uint32_t h[2], l[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float a = __uint_as_float(v[2 * k]), b = __uint_as_float(v[2 * k + 1]);
        h[k] = __builtin_bit_cast(uint32_t, half2v{(_Float16)(a * scale), (_Float16)(b * scale)});
        asm("" : "+v"(h[k]));                       // (as it is: both halves are read from here, not rounded a second time)
        const half2v first = __builtin_bit_cast(half2v, h[k]);
        l[k] = __builtin_bit_cast(uint32_t, half2v{(_Float16)__builtin_fmaf(a, scale, -(float)first[0]), (_Float16)__builtin_fmaf(b, scale, -(float)first[1])});
    }
    *reinterpret_cast<uint2*>(high) = make_uint2(h[0], h[1]);
    *reinterpret_cast<uint2*>(low) = make_uint2(l[0], l[1]);
}

// Chunks of 128 k of a tile of 16 rows of weights, the last of which may be a part.  Kernels ask for them some chunks ahead, every lane for every chunk alike
// (a load that a branch may pass over makes the compiler wait for all of them), so what lies past the end of a row of K >= 128 is moved back into it:
//   codes   MXFP4: block 4 c + q, or the last one; NVFP4: blocks 8 c + 2 q and the next, or the last two
//   scales  the chunk's 4 or 8 bytes, or the last ones of the row
// and whole() puts right on arrival what was moved.  Codes of blocks past the end are those of some block; rows are zero there.  Addresses are a
// tile's, the same for all lanes, and a lane's offset, the same for all tiles and chunks.
template <int B>
struct Row {                                        // the lane's
    static constexpr int SB = 128 / B;              // scale bytes of a chunk
    uint32_t code, part, scale;                     // offsets of the codes of chunk 0 and of the part of a chunk, and of the scales
    int blocks, last;                               // of a row; the part's chunk
    bool odd;                                       // the lane's first block of the part is the row's last
    __device__ Row(int row, int q, int K, int64_t code_pitch, int64_t scale_pitch) {
        blocks = K / B;
        last = K >> 7;
        odd = 8 * last + 2 * q == blocks - 1;
        code = (uint32_t)row * (uint32_t)code_pitch + 16u * q;
        part = (uint32_t)row * (uint32_t)code_pitch + (uint32_t)(B == 16 ? 8 * min(8 * last + 2 * q, blocks - 2) : 16 * min(4 * last + q, blocks - 1));
        scale = (uint32_t)row * (uint32_t)scale_pitch;
    }
    __device__ u32x4 codes(const uint8_t* tile, int c) const {
        return *reinterpret_cast<const u32x4_a4*>(c == last ? tile + part : tile + 64 * c + code);
    }
    __device__ u32x2 scales(const uint8_t* tile, int c) const {
        const uint8_t* at = tile + (scale + (uint32_t)min(SB * c, blocks - SB));
        if constexpr (B == 16) {
            const uint2 v = load8_a1(at);
            return u32x2{v.x, v.y};
        } else {
            return u32x2{load4_a1(at), 0u};
        }
    }
    // the chunk's scale bytes in their places; of a whole chunk nothing changes
    __device__ u32x2 whole(u32x2 s, int c) const {
        const int off = 8 * max(SB * c - (blocks - SB), 0);
        if constexpr (B == 32) return u32x2{s[0] >> off | (0x70707070u & ~(0xFFFFFFFFu >> off)), 0u};       // (bytes past the end that fold)
        const uint64_t v = ((uint64_t)s[1] << 32 | s[0]) >> off;
        return u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
    }
    // and its codes: NVFP4's last block may be the second of two that were read
    __device__ uint4 whole(u32x4 v, int c) const {
        if constexpr (B == 32) return make_uint4(v[0], v[1], v[2], v[3]);
        const bool second = c == last && odd;
        return make_uint4(second ? v[2] : v[0], second ? v[3] : v[1], v[2], v[3]);
    }
    // those of a chunk's bytes that go with the lane's words, one for each
    __device__ static uint32_t of_lane(u32x2 s, int q) {
        return B == 16 ? __builtin_amdgcn_perm(s[1], s[0], q < 2 ? 0x06040200u : 0x07050301u) : s[0];
    }
};
// Where a tile starts whose first row is `row` of expert e (uniform).
__device__ __forceinline__ const uint8_t* codes_of(const Experts& w, int e, int64_t row) { return w.codes + ((int64_t)e * w.rows + row) * w.code_pitch; }
__device__ __forceinline__ const uint8_t* scales_of(const Experts& w, int e, int64_t row) { return w.scales + ((int64_t)e * w.rows + row) * w.scale_pitch; }

// `count` chunks whose scales do not all fold, asked for only here, one at a time: rows(d, fragments), codes(d, tile).
template <int B, int MT, int N, int NT, typename Rows, typename Codes>
__device__ __forceinline__ void block_by_block(int count, const uint32_t (&sw)[N][NT], const Rows& rows, const Codes& codes, float4v (&acc)[MT][NT]) {
    if constexpr (B == 32) {
#pragma unroll 1
        for (int d = 0; d < count; ++d) {
            half8 xf[MT][4];
            rows(d, xf);
            uint4 words[NT];
            uint32_t one[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                words[t] = codes(d, t);
                one[t] = d == 0 ? sw[0][t] : d == 1 ? sw[1][t] : d == 2 ? sw[2][t] : d == 3 ? sw[3][t] : sw[N - 1][t];
            }
            multiply_folded<B, false, MT>(xf, words, one, acc);
        }
    }
}

template <int MT, int NT>
__device__ __forceinline__ void clear(float4v (&acc)[MT][NT]) {
#pragma unroll
    for (int r = 0; r < MT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[r][t] = float4v{0.f, 0.f, 0.f, 0.f};
}

// ---- a few tokens: up to 64 slots, which a wave holds in its lanes

// The distinct experts of up to 64 slots, in the order in which they appear, in lanes 0 .. count - 1 of the result.  id: of the lane's slot, -1 for none.
__device__ __forceinline__ int distinct(int id, int& count) {
    const int lane = threadIdx.x & 63;
    int found = -1, n = 0;
    for (uint64_t left = __ballot(id >= 0); left != 0; ++n) {
        const int e = __builtin_amdgcn_readlane(id, (int)__builtin_ctzll(left));
        left &= ~__ballot(id == e);
        if (lane == n) found = e;
    }
    count = n;
    return found;
}
__device__ __forceinline__ int checked_id(const int32_t* ids, int t, int slots, int E) {
    const int e = t < slots ? ids[t] : -1;
    return e >= 0 && e < E ? e : -1;
}

// The same for up to 256 slots, all threads of a workgroup of 512: the experts to `found`.
__device__ __forceinline__ int distinct(const int16_t* ids, int slots, int16_t* found, int (&counts)[8]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e = tid < slots ? ids[tid] : -1;
    bool first = e >= 0;
    for (int g = 0; g <= min(tid | 63, slots - 1) >> 3; ++g) {      // eight ids a read
        const u32x4 v = *reinterpret_cast<const u32x4*>(ids + 8 * g);
#pragma unroll
        for (int k = 0; k < 8; ++k) first = first && !((int16_t)(k & 1 ? v[k >> 1] >> 16 : v[k >> 1]) == e && 8 * g + k < tid);
    }
    const uint64_t firsts = __ballot(first);
    if (lane == 0) counts[wave] = __popcll(firsts);
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < 8; ++w) {
        before += w < wave ? counts[w] : 0;
        all += counts[w];
    }
    if (first) found[before + __popcll(firsts & ((1ull << lane) - 1ull))] = (int16_t)e;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(all);
}

// All tokens are rows of one tile, for every expert, so no list of an expert's tokens is needed: what comes out for one that does not choose it is passed over.
// They lie in LDS.  A tile of 16 columns of an expert, that is 16 rows of G and of U, is for KW waves, which split K; workgroups, one on a compute unit, take
// such a tile for each of their 8 / KW teams after the other, and ask for the next one's weights while they multiply and add up this one's.
// G: chunks in flight (a ring of two such groups was no faster).  SLOTS: most slots, 64 (experts in a wave's lanes) or 256 (in LDS).
constexpr int kGathered = 2;                        // pieces of 8 values a thread, at most, where it puts x in order
struct UpFewLds {
    float sums[8][2][4][64];                        // wave, G or U, element, lane
    float weights[256], scales[256];                // of a slot: its weight (a token's first choice of an expert: all of them), and the tensor scale of its expert
    __attribute__((aligned(16))) int16_t ids[256];
    int16_t active[256];
    int8_t choice[256][16];                         // of an active expert and a token: the first of its choices that is this expert, -1 for none
    int counts[8];
};
template <int B, int KW, int G, int SLOTS>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 4))) void up_few_kernel(UpArgs a) {
    constexpr int TEAMS = 8 / KW;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    UpFewLds& l = *reinterpret_cast<UpFewLds*>(lds);
    uint8_t* xs = lds + sizeof(UpFewLds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    const int kw = wave % KW, team = wave / KW, slots = a.M * a.top;
    const int mine = SLOTS == 64 ? lane : tid;      // of the slots
    const int id = checked_id(a.ids, mine, slots, a.E);
    const float weight_of = mine < slots ? a.weights[mine] : 0.0f;
    const int chunks = (a.K + 127) >> 7, pieces = a.K >> 3, pitch = 256 * chunks + 16;      // (16 bytes more than whole chunks: rows spread over the banks)
    const float scale_of = B == 16 && id >= 0 ? a.up.tensor_scales[id] : 1.0f / kFolded<B>;
    constexpr int AT_ONCE = 8;                      // pieces of a thread on their way
    const int per_row = 16 * chunks, all_pieces = per_row * a.M;
    // few enough values are put in order here: asked for before the weights and written to LDS behind them
    u32x4 order[kGathered][2];
    uint16_t gathered[kGathered][8];
    if (a.perm) {
#pragma unroll
        for (int k = 0; k < kGathered; ++k) {
            const int p = min(tid + 512 * k, all_pieces - 1) % per_row;
#pragma unroll
            for (int h = 0; h < 2; ++h) order[k][h] = *reinterpret_cast<const u32x4*>(a.perm + 8 * min(p, pieces - 1) + 4 * h);
        }
#pragma unroll
        for (int k = 0; k < kGathered; ++k) {
            const uint16_t* row = a.x + min(tid + 512 * k, all_pieces - 1) / per_row * a.ldx;
#pragma unroll
            for (int v = 0; v < 8; ++v) gathered[k][v] = row[min(order[k][v >> 2][v & 3], (uint32_t)a.K - 1u)];        // (an unchecked perm may point outside)
        }
    }
    for (int u0 = a.perm ? all_pieces : tid; u0 < all_pieces; u0 += 512 * AT_ONCE) {    // (pieces past the end are zeros)
        u32x4 v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int u = min(u0 + 512 * k, all_pieces - 1), m = u / per_row, p = u - m * per_row;
            v[k] = *reinterpret_cast<const u32x4*>(a.x + m * a.ldx + 8 * min(p, pieces - 1));
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int u = u0 + 512 * k, m = u / per_row, p = u - m * per_row;
            if (u < all_pieces) *reinterpret_cast<u32x4*>(xs + m * pitch + 16 * p) = p < pieces ? v[k] : u32x4{0, 0, 0, 0};
        }
    }
    if (tid < SLOTS) {
        l.ids[tid] = (int16_t)id;
        l.weights[tid] = weight_of;
        l.scales[tid] = scale_of;
    }
    int actives, active = -1;
    if constexpr (SLOTS == 64) {
        active = distinct(id, actives);
    } else {
        __syncthreads();
        actives = distinct(l.ids, slots, l.active, l.counts);
    }
    auto expert_of = [&](int nth) { return SLOTS == 64 ? __builtin_amdgcn_readlane(active, nth) : __builtin_amdgcn_readfirstlane(l.active[nth]); };
    const int all = actives * a.tiles, stride = (int)gridDim.x * TEAMS;
    const Row<B> of(i, q, a.K, a.up.code_pitch, a.up.scale_pitch);
    const uint8_t* x_lane = xs + min(i, a.M - 1) * pitch + 16 * q;
    const int c0 = kw * chunks / KW, n = (kw + 1) * chunks / KW - c0, groups = (n + G - 1) / G;     // n >= 1
    const uint8_t *wc[2], *ws[2];
    auto take = [&](int item) {                     // the item whose weights are asked for next
        const int nth = item / a.tiles, e = expert_of(nth);
#pragma unroll
        for (int t = 0; t < 2; ++t) {               // (I is a multiple of 16)
            wc[t] = codes_of(a.up, e, t * a.I + 16 * (item - nth * a.tiles));
            ws[t] = scales_of(a.up, e, t * a.I + 16 * (item - nth * a.tiles));
        }
    };
    u32x4 cw[G][2];
    u32x2 sc[2], fifth[2];
    auto ask_scales = [&](int g) {                  // lane group q: of the q-th chunk of the group; all lanes: of a fifth one
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = of.scales(ws[t], c0 + min(G * g + q, n - 1));
            if (G == 5) fifth[t] = of.scales(ws[t], c0 + min(G * g + 4, n - 1));
        }
    };
    auto ask_codes = [&](int g, int d) {
#pragma unroll
        for (int t = 0; t < 2; ++t) cw[d][t] = of.codes(wc[t], c0 + min(G * g + d, n - 1));
    };
    int item = (int)blockIdx.x * TEAMS + team;
    const int rounds = (all - (int)blockIdx.x * TEAMS + stride - 1) / stride;       // of the workgroup's first team: the others have as many, or one fewer
    if (rounds <= 0) return;
    take(min(item, all - 1));                       // (a team without work asks for the last item's)
    ask_scales(0);
#pragma unroll
    for (int d = 0; d < G; ++d) ask_codes(0, d);
    if (a.perm) {
#pragma unroll
        for (int k = 0; k < kGathered; ++k) {
            const int u = tid + 512 * k, m = u / per_row, p = u - m * per_row;
            u32x4 v = {0, 0, 0, 0};
            if (p < pieces)
#pragma unroll
                for (int h = 0; h < 4; ++h) v[h] = (uint32_t)gathered[k][2 * h] | (uint32_t)gathered[k][2 * h + 1] << 16;
            if (u < all_pieces) *reinterpret_cast<u32x4*>(xs + m * pitch + 16 * p) = v;
        }
    }
    wait_lgkmcnt0();
    wg_barrier();                                   // not __syncthreads(): the weights stay in flight
    // which token chooses which expert, once and not for every tile; what is written here is read behind the first round's barriers
    for (int k0 = 64 * wave; k0 < 16 * actives; k0 += 512) {
        const int nth = (k0 + lane) >> 4, m = lane & 15;
        const int e = SLOTS == 64 ? __shfl(active, nth & 63) : l.active[min(nth, actives - 1)];        // (every lane takes part)
        int choice = -1;
        float weight = 0.0f;
        if (m < a.M && nth < actives) {
            for (int j = 0; j < a.top; ++j)
                if (l.ids[m * a.top + j] == e) {
                    choice = choice < 0 ? j : choice;
                    weight += l.weights[m * a.top + j];
                }
            if (choice >= 0) l.weights[m * a.top + choice] = weight;
        }
        if (nth < actives) l.choice[nth][m] = (int8_t)choice;
    }
    for (int round = 0; round < rounds; ++round, item += stride) {
        float4v acc[1][2];
        clear<1, 2>(acc);
        for (int g = 0; g < groups; ++g) {
            const bool over = g + 1 == groups;
            const int count = min(G, n - G * g), next = over ? 0 : g + 1, c = c0 + G * g;
            uint32_t sw[G < 4 ? 4 : G][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u32x2 v = of.whole(sc[t], c0 + min(G * g + q, n - 1));
                uint32_t s[4];
                scales_of_group<B>(make_uint2(v[0], v[1]), s);
#pragma unroll
                for (int d = 0; d < 4; ++d) sw[d][t] = s[d];
                if constexpr (G == 5) sw[4][t] = of.of_lane(of.whole(fifth[t], c0 + min(G * g + 4, n - 1)), q);
            }
            auto rows_of = [&](int d, half8 (&xf)[1][4]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[0][j] = *reinterpret_cast<const half8*>(x_lane + 256 * (c + d) + 64 * j);
            };
            const bool fold = folds<B>(sw);
            if (!fold) block_by_block<B, 1>(count, sw, rows_of, [&](int d, int t) { return of.whole(of.codes(wc[t], c + d), c + d); }, acc);
            if (over) take(min(item + stride, all - 1));
            ask_scales(next);
            if (fold) {
#pragma unroll
                for (int d = 0; d < G; ++d) {
                    if (d < count) {                // (rows past the wave's last chunk are another's)
                        half8 xf[1][4];
                        rows_of(d, xf);
                        uint4 words[2];
#pragma unroll
                        for (int t = 0; t < 2; ++t) words[t] = of.whole(cw[d][t], c + d);
                        multiply_folded<B, true, 1>(xf, words, sw[d], acc);
                    }
                    ask_codes(next, d);
                }
            } else {
#pragma unroll
                for (int d = 0; d < G; ++d) ask_codes(next, d);
            }
        }
        if (round > 0) wg_barrier();                // (the sums of the round before have been read)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) l.sums[wave][t][k][lane] = acc[0][t][k];
        wait_lgkmcnt0();
        wg_barrier();
        if (item < all) {
            const int nth = item / a.tiles, n0 = 16 * (item - nth * a.tiles);
            for (int idx = kw * 64 + lane; idx < 16 * a.M; idx += 64 * KW) {
                const int m = idx >> 4, at = 16 * (m >> 2) + (idx & 15), k = m & 3;
                const int choice = l.choice[nth][m], slot = m * a.top + choice;
                if (choice < 0) continue;
                float g = 0.f, u = 0.f;
#pragma unroll
                for (int w = 0; w < KW; ++w) g += l.sums[team * KW + w][0][k][at], u += l.sums[team * KW + w][1][k][at];
                const float alpha = l.scales[slot];
                store_h(a, slot, n0 + (idx & 15), g * alpha, u * alpha, l.weights[slot]);
            }
        }
        wait_lgkmcnt0();                            // (reads of the sums have come back before the next barrier)
    }
}

// Up to 4 tokens: 16 columns of y a workgroup.  The reduction runs over all chosen experts' channels one after the other, in equal shares for the waves, G
// chunks at a time; a wave adds what it has of an expert to its own sums of all tokens, and the waves' sums are added in their order at the end.
// Rows of h reach a wave's registers through a slice of LDS of its own, so that a chunk on its way takes TOKENS / 2 registers of 16 bytes and not four.  A row
// of h has one unit, by the exponents that came with it: looking for the largest values of a chunk on its arrival instead took 2 to 10 % of a call.
constexpr int kFewTables = 256 + 512 + 256 + 256;      // bytes of its tables in LDS
template <int B, int TOKENS, int WAVES, typename OutT>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(4, 4))) void down_few_kernel(DownArgs<OutT> a) {
    constexpr int THREADS = 64 * WAVES, LOADS = TOKENS / 2, G = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float(&sums)[WAVES][8][16] = *reinterpret_cast<float(*)[WAVES][8][16]>(lds);
    int* ids_of = reinterpret_cast<int*>(lds + sizeof(sums));
    int8_t(&slot_of)[64][8] = *reinterpret_cast<int8_t(*)[64][8]>(lds + sizeof(sums) + 256);       // of an active expert and a token; -1: it does not choose it
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    float* scales_of_slots = reinterpret_cast<float*>(lds + sizeof(sums) + 256 + 512);
    uint32_t* exponents = reinterpret_cast<uint32_t*>(lds + sizeof(sums) + 256 + 512 + 256);
    uint8_t* slice = lds + sizeof(sums) + kFewTables + wave * TOKENS * 512;
    const int slots = a.M * a.top, id = checked_id(a.ids, lane, slots, a.E);
    const int row_bytes = exponents_pitch(a.I >> 4), exponent_pieces = slots * row_bytes >> 4;
    const u32x4 some = *reinterpret_cast<const u32x4*>(a.exponents + 16 * min(tid, exponent_pieces - 1));
    if (wave == 0) {
        exponents[lane] = kLeast;
        ids_of[lane] = id;
        scales_of_slots[lane] = B == 16 && id >= 0 ? a.down.tensor_scales[id] : 1.0f / kFolded<B>;
    }
    for (int k = lane; k < 128; k += 64) (&sums[wave][0][0])[k] = 0.0f;
    int actives;
    const int active = distinct(id, actives);
    __syncthreads();
    for (int k0 = 64 * wave; k0 < 8 * actives; k0 += THREADS) {
        const int nth = (k0 + lane) >> 3, m = lane & 7, e = __shfl(active, nth & 63);       // (every lane takes part)
        int slot = -1;
        if (m < a.M)
            for (int j = a.top - 1; j >= 0; --j) slot = ids_of[m * a.top + j] == e ? m * a.top + j : slot;
        if (nth < actives) slot_of[nth][m] = (int8_t)slot;
    }
    __syncthreads();
    const int n0 = (int)blockIdx.x * 16;
    const Row<B> of(min(i, a.N - 1 - n0), q, a.I, a.down.code_pitch, a.down.scale_pitch);
    const int per = (a.I + 127) >> 7, groups = (per + G - 1) / G, all = actives * groups;
    const int s0 = wave * all / WAVES, s1 = (wave + 1) * all / WAVES;
    // a load: a chunk of two tokens, 32 lanes each; in LDS rows r = 2 token + (0: first numbers, 1: second ones), in pieces of eight
    const int part = lane & 31, half = lane >> 5;
    auto unit = [](int piece, int r) { return 16 * (2 * TOKENS * piece + (r ^ (piece & (2 * TOKENS - 1)))); };
    const int to = unit(part >> 1, 2 * half) + 8 * (part & 1);
    const uint8_t *wc = nullptr, *ws = nullptr;
    uint32_t row[LOADS], chunk[LOADS];              // offsets from a.h, and what a chunk adds to them
    auto take = [&](int nth) {                      // the expert whose weights are asked for next
        const int e = __builtin_amdgcn_readlane(active, nth);
        wc = codes_of(a.down, e, n0);
        ws = scales_of(a.down, e, n0);
#pragma unroll
        for (int l = 0; l < LOADS; ++l) {           // (the row of a token that does not choose it is passed over: the same piece all the time)
            const int slot = slot_of[nth][2 * l + half];
            row[l] = slot < 0 ? 0u : (uint32_t)slot * (uint32_t)a.pitch + 4u * part;
            chunk[l] = slot < 0 ? 0u : 128u;
        }
    };
    u32x4 cw[G], rows[G][LOADS];
    u32x2 sc;
    auto ask_scales = [&](int g) { sc = of.scales(ws, min(G * g + q, per - 1)); };
    auto load_rows = [&](int c, u32x4 (&to)[LOADS]) {
#pragma unroll
        for (int l = 0; l < LOADS; ++l) to[l] = *reinterpret_cast<const u32x4*>(a.h + (row[l] + chunk[l] * (uint32_t)c));
    };
    auto ask_chunk = [&](int g, int d) {
        const int c = min(G * g + d, per - 1);
        load_rows(c, rows[d]);
        cw[d] = of.codes(wc, c);
    };
    int nth = s0 / max(groups, 1), g = s0 - nth * groups;
    if (s0 < s1) {
        take(nth);
        ask_scales(g);
#pragma unroll
        for (int d = 0; d < G; ++d) ask_chunk(g, d);
    }
    // the rows' units, while weights are on their way
    auto count_exponents = [&](int u, const u32x4& v) { atomicMax(&exponents[(u << 4) / row_bytes], min(largest_byte(v), kMost)); };
    if (tid < exponent_pieces) count_exponents(tid, some);
    for (int u = tid + THREADS; u < exponent_pieces; u += THREADS) count_exponents(u, *reinterpret_cast<const u32x4*>(a.exponents + 16 * u));
    wait_lgkmcnt0();
    wg_barrier();
    if (s0 < s1) {
        float scale[LOADS];                         // to the rows' units
        auto take_units = [&](int nth) {
#pragma unroll
            for (int l = 0; l < LOADS; ++l) scale[l] = scale_to(exponents[max((int)slot_of[nth][2 * l + half], 0)]);
        };
        take_units(nth);
        float4v acc[1][1];
        clear<1, 1>(acc);
        for (int s = s0; s < s1; ++s) {
            const int count = min(G, per - G * g);
            const bool over = g + 1 == groups, end = s + 1 == s1;
            const int next = end ? g : over ? 0 : g + 1;        // (behind the last one: itself again)
            const u32x2 v = of.whole(sc, min(G * g + q, per - 1));
            uint32_t one[4], sw[4][1];
            scales_of_group<B>(make_uint2(v[0], v[1]), one);
#pragma unroll
            for (int d = 0; d < 4; ++d) sw[d][0] = one[d];
            auto rows_of = [&](const u32x4 (&from)[LOADS], half8 (&xf)[1][4]) {     // (LDS operations of a wave complete in order)
#pragma unroll
                for (int l = 0; l < LOADS; ++l) {   // (token 2 l and its second row by exclusive or: neither changes another bit of the place)
                    const int at = to ^ 64 * l;
                    put_h(from[l], scale[l], slice + at, slice + (at ^ 16));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[0][j] = *reinterpret_cast<const half8*>(slice + unit(4 * j + q, 2 * (i & (TOKENS - 1)) + (i >> 3)));
            };
            const bool fold = folds<B>(sw);
            if (!fold)
                block_by_block<B, 1>(count, sw, [&](int d, half8 (&xf)[1][4]) {
                    u32x4 from[LOADS];
                    load_rows(G * g + d, from);
                    rows_of(from, xf);
                }, [&](int d, int) { return of.whole(of.codes(wc, G * g + d), G * g + d); }, acc);
            if (over && !end) take(nth + 1);
            ask_scales(next);
            if (fold) {
#pragma unroll
                for (int d = 0; d < G; ++d) {
                    if (d < count) {
                        half8 xf[1][4];
                        rows_of(rows[d], xf);
                        uint4 words[1] = {of.whole(cw[d], G * g + d)};
                        multiply_folded<B, true, 1>(xf, words, sw[d], acc);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    ask_chunk(next, d);
                }
            } else {
#pragma unroll
                for (int d = 0; d < G; ++d) ask_chunk(next, d);
            }
            if (over || end) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // lanes of the first half hold sums of first numbers, those of the second of second ones of the same rows
                    const uint2v both = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[0][0][k]), __float_as_uint(acc[0][0][k]), false, false);
                    const float sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
                    const int slot = lane < 32 ? slot_of[nth][4 * q + k] : -1;
                    if (slot >= 0) sums[wave][4 * q + k][i] += sum * scale_from(exponents[slot]) * scales_of_slots[slot];
                }
                clear<1, 1>(acc);
                ++nth;
                if (!end) take_units(nth);
            }
            g = next;
        }
    }
    __syncthreads();
    for (int idx = tid; idx < a.M * 16; idx += THREADS) {
        const int m = idx >> 4, n = n0 + (idx & 15);
        if (n >= a.N) continue;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += sums[w][m][idx & 15];
        if (a.residual) sum += (float)a.residual[m * a.ldr + n];
        store_out(a.y + m * a.ldy + n, sum);
    }
}

// ---- more tokens: rows gathered by expert

// Which slots (token, choice) every expert has, in blocks of up to ROWS.
struct Lists {
    uint16_t start[kMostExperts], count[kMostExperts];
    uint16_t slots[kMostSlots];                 // by expert
    int16_t id[kMostSlots];                     // by slot, -1 for none
    __attribute__((aligned(16))) int16_t first[kMostSlots];      // the same without a token's later choices of an expert: those count with the first
    uint16_t expert[kMostSlots], begin[kMostSlots];     // of a block: its expert, and the first of that expert's slots
    uint32_t fill[kMostExperts];
    float weight[kMostSlots];                   // by slot, where asked for: all that a token's choices of an expert weigh, at the first
    int blocks;
};
constexpr size_t kListBytes = (sizeof(Lists) + 15) / 16 * 16;

// Of a value a lane: the sum over the lanes before.
__device__ __forceinline__ int sum_before(int n) {
    const int lane = threadIdx.x & 63;
    int sum = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    return sum - n;
}

// All threads of the workgroup.  An expert's slots are in ascending order: every workgroup has the same blocks.  weights: or null
template <int THREADS, int ROWS>
__device__ void lists_of(const int32_t* __restrict__ ids, const float* __restrict__ weights, int M, int top, int E, Lists& l) {
    const int tid = threadIdx.x, slots = M * top;
    constexpr int PER = (kMostSlots + THREADS - 1) / THREADS;
    int id[PER], at[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = tid + p * THREADS;
        id[p] = checked_id(ids, t, slots, E);
        if (t < kMostSlots) l.id[t] = (int16_t)id[p];
    }
    for (int e = tid; e < E; e += THREADS) l.fill[e] = 0;
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = tid + p * THREADS;
        for (int u = t - t % top; u < t && id[p] >= 0; ++u)
            if (l.id[u] == id[p]) id[p] = -1;
        if (t < kMostSlots) l.first[t] = (int16_t)id[p];
        if (id[p] >= 0) atomicAdd(&l.fill[id[p]], 1u);
        if (id[p] >= 0 && weights) {
            float weight = weights[t];
            for (int u = t + 1; u < t - t % top + top; ++u)
                if (l.id[u] == id[p]) weight += weights[u];
            l.weight[t] = weight;
        }
    }
    __syncthreads();
    // a slot's place: how many before it have its expert, eight ids a read
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        const int t = tid + p * THREADS, until = min(t | 63, slots - 1) >> 3;
        at[p] = 0;
        if (p * THREADS >= slots) continue;
        for (int g = 0; g <= until; ++g) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(l.first + 8 * g);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int other = (int16_t)(k & 1 ? v[k >> 1] >> 16 : v[k >> 1]);
                at[p] += other == id[p] && 8 * g + k < t ? 1 : 0;
            }
        }
    }
    if (tid < 64) {
        int begin = 0, blocks = 0;
        for (int base = 0; base < E; base += 64) {
            const int e = base + tid, n = e < E ? (int)l.fill[e] : 0, mine = (n + ROWS - 1) / ROWS;
            const int before = begin + sum_before(n), block = blocks + sum_before(mine);
            if (e < E) {
                l.start[e] = (uint16_t)before;
                l.count[e] = (uint16_t)n;
            }
            for (int k = 0; k < mine; ++k) {
                l.expert[block + k] = (uint16_t)e;
                l.begin[block + k] = (uint16_t)(ROWS * k);
            }
            begin = __shfl(before + n, 63);
            blocks = __shfl(block + mine, 63);
        }
        if (tid == 0) l.blocks = blocks;
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < PER; ++p)
        if (id[p] >= 0) l.slots[l.start[id[p]] + at[p]] = (uint16_t)(tid + p * THREADS);
    __syncthreads();
}

// Where an item is: blocks of an expert over the same weights are next to each other, so that those come from memory once.
struct Place {
    int expert, first, left, piece;             // the first of the expert's slots in the list, and how many from there on; which of `pieces` pieces of its weights
};
template <int ROWS>
__device__ __forceinline__ Place place_of(const Lists& l, int item, int pieces) {
    const int some = item / pieces, e = __builtin_amdgcn_readfirstlane(l.expert[some]), begin = __builtin_amdgcn_readfirstlane(l.begin[some]);
    const int count = __builtin_amdgcn_readfirstlane(l.count[e]), start = __builtin_amdgcn_readfirstlane(l.start[e]);
    const int blocks = (count + ROWS - 1) / ROWS, local = item - (some - begin / ROWS) * pieces, piece = local / blocks, r0 = (local - piece * blocks) * ROWS;
    return {e, start + r0, count - r0, piece};
}

// A workgroup's piece of work: a block of an expert's slots with the eight waves' tiles of weights, two each, over a run of the reduction.
template <typename T>
struct Item {
    const T* from;                              // the row that this thread copies pieces of 16 bytes of
    const uint8_t *wc[2], *ws[2];               // the wave's tiles
    float scale;                                // of the weights
    int c0, c1;                                 // chunks
    bool two;                                   // rows behind the first 16 are in use
    Place place;
};

// Items of a launch in turn.  Rows reach all waves through LDS, kStage chunks at a time in two buffers: a barrier a stage.  (With 16 rows half of the threads copy
// every other chunk.)  Rows and weights of the next stage, or of the next item's first, are asked for in this one, rows first: they are needed first, and
// loads return in order.  take(n): the n-th; store(its place, its scale, sums).
// T: rows of fp16, 16 MT of them; or of fp32, 8 MT, each as two of fp16, rows r and r + 8 of a tile, in a unit that goes by the largest value so far.
// 32 rows an item (16 slots behind the activation): with 16, two workgroups a compute unit, 64 tokens of eight of 64 experts took 113 us and not 100; with 64,
// 64 tokens of two of eight 1.5 % less, 32 tokens 2 % more, since the rows' matrix work and reads of LDS are what an item's time is then.
constexpr int kStage = 4;
template <int MT>
constexpr int kRowBytes = kStage * MT * 4096;   // of a buffer

// Which row a thread copies pieces of, and which of a chunk's pieces of 16 bytes: rows of fp32 have 32, so that half a wave has all of a row's.
template <typename T, int MT>
__device__ __forceinline__ int copied_row() {
    if (std::is_same<T, float>::value) return MT == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : (int)threadIdx.x / (64 / MT);
    return (int)(threadIdx.x >> 4) & (16 * MT - 1);
}

template <int B, int MT, typename T, typename Take, typename Store>
__device__ __forceinline__ void stream_items(int begin, int end, int stride, const Row<B>& of, int K, uint8_t* lds, float (*units)[2][8 * MT], const Take& take, const Store& store) {
    constexpr bool SPLIT = std::is_same<T, float>::value;
    constexpr int G = kStage, PER = 2 * MT, NT = 2; // pieces of a thread
    constexpr int OF_PIECE = 16 / (int)sizeof(T), PIECES = 128 / OF_PIECE;      // values of a piece, pieces of a chunk's row
    const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, q = lane >> 4;
    const int piece = tid & (PIECES - 1), pieces = K / OF_PIECE, blocks = of.blocks, row = copied_row<T, MT>();
    auto chunk_of = [&](int k) { return MT == 2 ? k : 2 * k + (SPLIT ? lane >> 5 : tid >> 8); };
    auto unit = [](int p, int r) { return 16 * (256 * (r >> 4) + 16 * p + ((r & 15) ^ p)); };
    const int to = SPLIT ? unit(piece >> 1, 16 * (row >> 3) + (row & 7)) + 8 * (piece & 1) : unit(piece, row);
    // N pieces of the thread's row, of chunks chunk_of(0 ..); all threads of a wave.  SPLIT: a row's unit only grows from the item's first stage on; left for whoever
    // has the sums: what they are multiplied by before this stage's are added, and what takes them back.
    uint32_t most = kLeast;
    auto put = [&](auto& v, int buffer, bool first) {
        constexpr int N = sizeof(v) / sizeof(v[0]);
        uint8_t* at = lds + buffer * kRowBytes<MT>;
        if constexpr (SPLIT) {
            float largest = 0.0f;
#pragma unroll
            for (int k = 0; k < N; ++k) largest = __builtin_elementwise_maximum(largest, magnitude(v[k]));
            uint32_t stage = half_wave_max(__float_as_uint(largest));
            if constexpr (MT == 1) {                // (a wave has a row)
                const uint2v halves = __builtin_amdgcn_permlane32_swap(stage, stage, false, false);
                stage = max(halves[0], halves[1]);
            }
            stage = min(max(stage >> 23, kLeast), kMost);
            const uint32_t before = first ? stage : most;
            most = max(before, stage);
            if (piece == 0) {
                units[buffer][0][row] = most - before < 127 ? __uint_as_float((127 - (most - before)) << 23) : 0.0f;
                units[buffer][1][row] = scale_from(most);
            }
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (N > 1 || chunk_of(k) == 0) put_h(v[k], scale_to(most), at + chunk_of(k) * MT * 4096 + to, at + chunk_of(k) * MT * 4096 + (to ^ 128));       // (eight rows on)
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (N > 1 || chunk_of(k) == 0) *reinterpret_cast<u32x4*>(at + chunk_of(k) * MT * 4096 + to) = v[k];
        }
    };
    auto multiply_by = [&](const float (&scales)[8 * MT], float4v (&acc)[MT][NT]) {
#pragma unroll
        for (int r = 0; r < MT; ++r) {
            const float4v scale = *reinterpret_cast<const float4v*>(&scales[8 * r + 4 * (q & 1)]);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[r][t][k] *= scale[k];
        }
    };
    if (begin >= end) return;
    if (blocks < of.SB) {                           // less than one chunk: too short to be moved back into
        for (int item = begin; item < end; item += stride) {
            const Item<T> now = take(item);
            u32x4 one[1] = {{0, 0, 0, 0}};
            if (chunk_of(0) == 0 && piece < pieces) one[0] = *reinterpret_cast<const u32x4*>(now.from + OF_PIECE * piece);
            put(one, 0, true);
            uint4 words[NT];
            uint32_t sw[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                u32x4 v = {0, 0, 0, 0};
                uint64_t s = 0;
                if constexpr (B == 16) {
                    if (2 * q < blocks) {
                        const uint2 w = load8_a8(now.wc[t] + of.code);
                        v[0] = w.x, v[1] = w.y;
                    }
                    if (2 * q + 1 < blocks) {
                        const uint2 w = load8_a8(now.wc[t] + of.code + 8);
                        v[2] = w.x, v[3] = w.y;
                    }
                } else {
                    if (q < blocks) v = *reinterpret_cast<const u32x4_a4*>(now.wc[t] + of.code);
                }
                for (int k = 0; k < blocks; ++k) s |= (uint64_t)now.ws[t][of.scale + k] << (8 * k);
                words[t] = make_uint4(v[0], v[1], v[2], v[3]);
                sw[t] = of.of_lane(u32x2{(uint32_t)s, (uint32_t)(s >> 32)}, q);
            }
            __syncthreads();
            half8 xf[MT][4];
            float4v acc[MT][NT];
            clear<MT, NT>(acc);
#pragma unroll
            for (int r = 0; r < MT; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j) xf[r][j] = *reinterpret_cast<const half8*>(lds + unit(4 * j + q, 16 * r + i));
            multiply_folded<B, B == 16, MT>(xf, words, sw, acc);
            if constexpr (SPLIT) multiply_by(units[0][1], acc);
            store(now.place, now.scale, acc);
            __syncthreads();
        }
        return;
    }
    u32x4 rows[PER], cw[G][NT];
    u32x2 sc[NT];
    Item<T> ahead = take(begin);                    // whose loads are asked for next
    auto ask_rows = [&](int c) {                    // (past the end: the last chunk again)
#pragma unroll
        for (int k = 0; k < PER; ++k)
            rows[k] = *reinterpret_cast<const u32x4*>(ahead.from + OF_PIECE * min(PIECES * min(c + chunk_of(k), ahead.c1 - 1) + piece, pieces - 1));
    };
    auto put_rows = [&](int c, int buffer) {
        u32x4 v[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const bool in = c + chunk_of(k) < ahead.c1 && PIECES * (c + chunk_of(k)) + piece < pieces;      // (all four chunks are multiplied)
            v[k] = in ? rows[k] : u32x4{0, 0, 0, 0};
        }
        put(v, buffer, c == ahead.c0);
    };
    auto ask_scales = [&](int c) {                  // lane group q: of chunk c + q
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t] = of.scales(ahead.ws[t], min(c + q, ahead.c1 - 1));
    };
    auto ask_codes = [&](int d, int c) {
#pragma unroll
        for (int t = 0; t < NT; ++t) cw[d][t] = of.codes(ahead.wc[t], min(c + d, ahead.c1 - 1));
    };
    ask_rows(ahead.c0);
    ask_scales(ahead.c0);
#pragma unroll
    for (int d = 0; d < G; ++d) ask_codes(d, ahead.c0);
    put_rows(ahead.c0, 0);
    wait_lgkmcnt0();
    wg_barrier();
    int buffer = 0;
    for (int item = begin; item < end; item += stride) {
        const int c0 = ahead.c0, c1 = ahead.c1;
        const bool two = ahead.two;
        const float scale = ahead.scale;
        const Place place = ahead.place;
        Item<T> after;                              // found out where loads are on their way, not where some are to be asked for
        bool known = false;
        float4v acc[MT][NT];
        clear<MT, NT>(acc);
        for (int c = c0; c < c1; c += G) {
            if constexpr (SPLIT)
                if (c != c0) multiply_by(units[buffer][0], acc);
            uint32_t sw[4][NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const u32x2 v = of.whole(sc[t], min(c + q, c1 - 1));
                uint32_t one[4];
                scales_of_group<B>(make_uint2(v[0], v[1]), one);
#pragma unroll
                for (int d = 0; d < 4; ++d) sw[d][t] = one[d];
            }
            auto rows_of = [&](int d, auto& xf, auto tiles) {
                const uint8_t* at = lds + buffer * kRowBytes<MT> + d * MT * 4096;
#pragma unroll
                for (int r = 0; r < decltype(tiles)::value; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) xf[r][j] = *reinterpret_cast<const half8*>(at + unit(4 * j + q, 16 * r + i));
            };
            using All = std::integral_constant<int, MT>;
            const bool fold = folds<B>(sw);
            if (!fold)
                block_by_block<B, MT>(min(G, c1 - c), sw, [&](int d, half8 (&xf)[MT][4]) { rows_of(d, xf, All{}); },
                                      [&](int d, int t) { return of.whole(of.codes(ahead.wc[t], c + d), c + d); }, acc);
            int next = c + G;
            if (next >= c1) {
                ahead = known ? after : take(item + stride < end ? item + stride : item);
                next = ahead.c0;
            }
            ask_rows(next);
            ask_scales(next);
            if (MT > 1 && c == c0 && c + G < c1) {      // (with MT = 1 registers do not allow it)
                after = take(item + stride < end ? item + stride : item);
                known = true;
            }
            auto multiply = [&](auto tiles) {
#pragma unroll
                for (int d = 0; d < G; ++d) {
                    half8 xf[MT][4];
                    rows_of(d, xf, tiles);
                    uint4 words[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) words[t] = of.whole(cw[d][t], c + d);
                    multiply_folded<B, true, decltype(tiles)::value>(xf, words, sw[d], acc);
                    ask_codes(d, next);
                }
            };
            if (!fold) {
#pragma unroll
                for (int d = 0; d < G; ++d) ask_codes(d, next);
            } else if (MT > 1 && !two) {
                multiply(std::integral_constant<int, 1>{});
            } else {
                multiply(All{});
            }
            if constexpr (SPLIT)
                if (c + G >= c1) multiply_by(units[buffer][1], acc);
            buffer ^= 1;
            put_rows(next, buffer);
            wait_lgkmcnt0();
            wg_barrier();                           // not __syncthreads(): loads stay in flight
        }
        store(place, scale, acc);
    }
}

// Items of a workgroup: those of an expert are next to each other, and workgroups of one XCD, which share an L2, take a run of them in turn.
struct Share {
    int begin, end, stride;
};
__device__ __forceinline__ Share share_of(int all) {
    constexpr int XCDS = 8;
    const int wg = (int)blockIdx.x, wgs = (int)gridDim.x, x = wg % XCDS, of_xcd = (wgs - x + XCDS - 1) / XCDS;
    const int x0 = (int)((int64_t)x * all / XCDS), x1 = (int)((int64_t)(x + 1) * all / XCDS);
    if (wgs < XCDS) return {wg, all, wgs};
    return {x0 + wg / XCDS, x1, of_xcd};
}

// An item: 128 columns of an expert for up to 16 MT of its tokens; a wave has 16 rows of G and of U.
template <int B, int MT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(MT == 1 ? 4 : 2, 4))) void up_many_kernel(UpArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Lists& l = *reinterpret_cast<Lists*>(lds + 2 * kRowBytes<MT>);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    lists_of<512, 16 * MT>(a.ids, a.weights, a.M, a.top, a.E, l);
    const int groups = (a.tiles + 7) >> 3, chunks = (a.K + 127) >> 7;
    const Row<B> of(i, q, a.K, a.up.code_pitch, a.up.scale_pitch);
    auto tile_of = [&](int group) { return min(8 * group + wave, a.tiles - 1); };       // (waves past the last tile repeat it)
    auto take = [&](int item) {
        const Place at = place_of<16 * MT>(l, item, groups);
        const int e = at.expert, left = at.left, tile = tile_of(at.piece);
        Item<uint16_t> v;
        v.from = a.x + (int64_t)(l.slots[at.first + min(copied_row<uint16_t, MT>(), left - 1)] / a.top) * a.ldx;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            v.wc[t] = codes_of(a.up, e, t * a.I + 16 * tile);
            v.ws[t] = scales_of(a.up, e, t * a.I + 16 * tile);
        }
        v.scale = B == 16 ? a.up.tensor_scales[e] : 1.0f / kFolded<B>;
        v.c0 = 0, v.c1 = chunks;
        v.two = left > 16;
        v.place = at;
        return v;
    };
    auto store = [&](const Place& place, float alpha, const float4v (&acc)[MT][2]) {
        const int left = place.left, first = place.first, tile = tile_of(place.piece);
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = 16 * r + 4 * q + k;
                if (at >= left) continue;
                const int slot = l.slots[first + at];
                store_h(a, slot, 16 * tile + i, acc[r][0][k] * alpha, acc[r][1][k] * alpha, l.weight[slot]);
            }
    };
    const Share mine = share_of(l.blocks * groups);
    stream_items<B, MT, uint16_t>(mine.begin, mine.end, mine.stride, of, a.K, lds, nullptr, take, store);
}

// Results of every slot by itself, in fp32.  An item: 256 columns of an expert over one of `splits` runs of I, for up to 8 MT of its tokens; a wave has 32 columns.
template <int B, int MT, typename OutT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(MT == 1 ? 4 : 2, 4))) void down_many_kernel(DownArgs<OutT> a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Lists& l = *reinterpret_cast<Lists*>(lds + 2 * kRowBytes<MT>);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
    float(*units)[2][8 * MT] = reinterpret_cast<float(*)[2][8 * MT]>(lds + 2 * kRowBytes<MT> + kListBytes);
    lists_of<512, 8 * MT>(a.ids, nullptr, a.M, a.top, a.E, l);
    const int chunks = (a.I + 127) >> 7, pieces = a.groups * a.splits, last = a.N < 16 ? 0 : a.N - 16;
    const Row<B> of(min(i, a.N - 1), q, a.I, a.down.code_pitch, a.down.scale_pitch);
    auto col_of = [&](int group) { return 32 * (8 * group + wave); };
    auto take = [&](int item) {
        const Place at = place_of<8 * MT>(l, item, pieces);
        const int e = at.expert, left = at.left, split = at.piece / a.groups, n0 = col_of(at.piece - split * a.groups);
        Item<float> v;
        v.from = a.h + (int64_t)l.slots[at.first + min(copied_row<float, MT>(), left - 1)] * a.pitch;
#pragma unroll
        for (int t = 0; t < 2; ++t) {               // tiles past the last column begin 16 before it; what an earlier tile has, too, is not stored
            v.wc[t] = codes_of(a.down, e, min(n0 + 16 * t, last));
            v.ws[t] = scales_of(a.down, e, min(n0 + 16 * t, last));
        }
        v.c0 = split * chunks / a.splits, v.c1 = (split + 1) * chunks / a.splits;
        v.scale = B == 16 ? a.down.tensor_scales[e] : 1.0f / kFolded<B>;
        v.two = left > 8;
        v.place = at;
        return v;
    };
    auto store = [&](const Place& place, float alpha, const float4v (&acc)[MT][2]) {
        const int left = place.left, first = place.first, split = place.piece / a.groups, n0 = col_of(place.piece - split * a.groups);
        float* out = a.partial + (int64_t)split * a.M * a.top * a.N;
#pragma unroll
        for (int r = 0; r < MT; ++r)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = 8 * r + 4 * (q & 1) + k;
                float* to = out + (int64_t)l.slots[first + min(at, left - 1)] * a.N;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint2v both = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[r][t][k]), __float_as_uint(acc[r][t][k]), false, false);
                    const float v = __uint_as_float(both[0]) + __uint_as_float(both[1]);
                    const int n = min(n0 + 16 * t, last) + i;
                    if (lane < 32 && at < left && n >= n0 + 16 * t && n < a.N) to[n] = v * alpha;
                }
            }
    };
    const Share mine = share_of(l.blocks * pieces);
    stream_items<B, MT, float>(mine.begin, mine.end, mine.stride, of, a.I, lds, units, take, store);
}

// y of a token: its slots' results, each over its runs, in their order, and the residual.
template <typename OutT>
__global__ __launch_bounds__(256) void join_kernel(DownArgs<OutT> a, uint32_t parts) {
    const int m = (int)(blockIdx.x / parts), n = (int)(blockIdx.x % parts) * 256 + (int)threadIdx.x;
    if (n >= a.N) return;
    float sum = 0.0f;
    for (int j = 0; j < a.top; ++j) {
        const int slot = m * a.top + j, e = a.ids[slot];
        bool counts = e >= 0 && e < a.E;
        for (int u = 0; u < j; ++u) counts = counts && a.ids[m * a.top + u] != e;       // (a later choice of the same expert counts with the first)
        if (!counts) continue;
        for (int s = 0; s < a.splits; ++s) sum += a.partial[((int64_t)s * a.M * a.top + slot) * a.N + n];
    }
    if (a.residual) sum += (float)a.residual[m * a.ldr + n];
    store_out(a.y + m * a.ldy + n, sum);
}

// Whether a launch's tokens go as rows of one tile: up to the activation wherever 16 rows and LDS take them, behind it up to 4 tokens.  Measured, us of a call, and with
// the tokens gathered instead in front of the activation, and behind it:
//                                            1 token        4 tokens          5 tokens          8 tokens          16 tokens
//   2048 x 1024, eight of 64, MXFP4        18.7  28  29      41   43   40      50    -   45      64   73   56       69   72
//   4096 x 14336, two of eight, NVFP4      52.7  59  60     142  176  148     160    -  153     193  219  175      182  204
//   4096 x 1792, eight of 128, MXFP4       31.9  44  44      87   99   90     110    -  107     165  175  152      239  240
//   5120 x 1392, four of 30, NVFP4, fp32   23.6  58  33      62   76   63      68    -   69      79   90   79      110  110
size_t up_few_lds(int64_t M, int64_t K) { return sizeof(UpFewLds) + (size_t)M * (size_t)((K + 127) / 128 * 256 + 16); }
bool up_few(int64_t M, int64_t top, int64_t K) { return M <= 16 && M * top <= 256 && K >= 256 && up_few_lds(M, K) <= kMaxLdsBytes; }
bool down_few(int64_t M, int64_t I) { return M <= 4 && I >= 128; }

// Waves that split K in up_few_kernel: as many as have four chunks each.  Measured, us of a call, and with half and with twice as many: K = 2048, eight of 64, one token
// 18.3, 19.7, 18.9, four 40.6, 40.9, 44.0; K = 4096, two of eight, one token with eight waves 52.4, with four 56.2, four tokens 143, 151; K = 1024, eight of 64, four tokens with
// two waves 31.4, with four 32.7.  And how many chunks go together, so that few are asked for in vain where a wave's are not a multiple of that.  (13 x 5120 x 1392, four
// of 30: 5 chunks a wave go as five in 93 us, as four and one of four in 97.)
int waves_of(int chunks) { return chunks >= 32 ? 8 : chunks >= 16 ? 4 : 2; }
int group_of(int chunks, int waves) {
    const int most = (chunks + waves - 1) / waves;
    int best = 5;
    for (const int g : {4, 3})
        if ((most + g - 1) / g * g < (most + best - 1) / best * best) best = g;
    return best;
}

// Runs of I for down_many_kernel: two items a compute unit, eight chunks in each at least.
constexpr int64_t kRunItems = 512;
int64_t most_runs(int64_t I) { return std::min<int64_t>((I + 127) / 128 / 8, 8); }
int down_splits(int64_t M, int64_t top, int64_t E, int64_t I, int64_t N) {
    const int64_t groups = (N + 255) / 256 * std::min<int64_t>(E, M * top);
    return (int)std::max<int64_t>(1, std::min<int64_t>(kRunItems / std::max<int64_t>(groups, 1), most_runs(I)));
}

int64_t pitch_of(int64_t I) { return (I + 127) / 128 * 128; }

// Bytes of a launch's parts of the workspace.
struct MoeWorkspace {
    size_t reordered, h, partial;               // rows in the weights' order; h, and its exponents; slots' results
};
size_t whole_lines(int64_t bytes) { return ((size_t)bytes + 255) / 256 * 256; }
size_t partial_bytes(int64_t M, int64_t top, int64_t E, int64_t I, int64_t N) {
    return M == 0 || down_few(M, I) ? 0 : whole_lines((int64_t)down_splits(M, top, E, I, N) * M * top * N * 4);
}
MoeWorkspace workspace_of(int64_t M, int64_t top, int64_t K, int64_t I, int64_t N, int64_t E, bool reorder) {
    const int64_t exponents = down_few(M, I) ? M * top * exponents_pitch((int)(I / 16)) : 0;
    return {reorder ? whole_lines(M * K * 2) : 0, whole_lines(M * top * pitch_of(I) * 4 + exponents), partial_bytes(M, top, E, I, N)};
}

template <int B, int KW, int G, int SLOTS>
arcq_status launch_up_slots(const UpArgs& u, int64_t items, hipStream_t stream) {
    auto kern = up_few_kernel<B, KW, G, SLOTS>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    const int64_t teams = 8 / KW;
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min<int64_t>((items + teams - 1) / teams, num_cu())), dim3(512), up_few_lds(u.M, u.K), stream, u);
    return check_launch("up_few_kernel");
}
template <int B, int KW>
arcq_status launch_up_few(const UpArgs& u, int64_t items, hipStream_t stream) {
    const bool few = u.M * u.top <= 64;
    switch (group_of((u.K + 127) / 128, KW)) {
        case 3: return few ? launch_up_slots<B, KW, 3, 64>(u, items, stream) : launch_up_slots<B, KW, 3, 256>(u, items, stream);
        case 4: return few ? launch_up_slots<B, KW, 4, 64>(u, items, stream) : launch_up_slots<B, KW, 4, 256>(u, items, stream);
        default: return few ? launch_up_slots<B, KW, 5, 64>(u, items, stream) : launch_up_slots<B, KW, 5, 256>(u, items, stream);
    }
}

template <int B, int TOKENS, int WAVES, typename OutT>
arcq_status launch_down_waves(const DownArgs<OutT>& d, hipStream_t stream) {
    auto kern = down_few_kernel<B, TOKENS, WAVES, OutT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3((unsigned)((d.N + 15) / 16)), dim3(64 * WAVES), WAVES * (512 + TOKENS * 512) + kFewTables, stream, d);
    return check_launch("down_few_kernel");
}

// 16 waves a workgroup, one on a compute unit; where a last round of those would leave a quarter of the compute units' time idle, 8, of which two fit.
// (5120 features, 1392 channels, four of 30, us of a call with 8 and with 16: one token 24, 27; four 61, 66.)
template <int B, int TOKENS, typename OutT>
arcq_status launch_down_few(const DownArgs<OutT>& d, hipStream_t stream) {
    const int64_t tiles = (d.N + 15) / 16, cus = num_cu(), rounds = (tiles + cus - 1) / cus;
    return tiles > cus && 4 * tiles < 3 * rounds * cus ? launch_down_waves<B, TOKENS, 8>(d, stream) : launch_down_waves<B, TOKENS, 16>(d, stream);
}

// items: as many as there can be.
template <int B, int MT>
arcq_status launch_up_many(const UpArgs& u, int64_t items, hipStream_t stream) {
    auto kern = up_many_kernel<B, MT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min<int64_t>(items, num_cu() * (MT == 1 ? 2 : 1))), dim3(512), 2 * kRowBytes<MT> + kListBytes, stream, u);
    return check_launch("up_many_kernel");
}
template <int B, int MT, typename OutT>
arcq_status launch_down_many(const DownArgs<OutT>& d, int64_t items, hipStream_t stream) {
    auto kern = down_many_kernel<B, MT, OutT>;
    static std::atomic<uint64_t> lds_raised{0};
    if (arcq_status st = raise_lds_limit(reinterpret_cast<const void*>(kern), lds_raised)) return st;
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min<int64_t>(items, num_cu() * (MT == 1 ? 2 : 1))), dim3(512), 2 * kRowBytes<MT> + kListBytes + 2 * 2 * 8 * MT * sizeof(float), stream, d);
    return check_launch("down_many_kernel");
}

template <int B, typename OutT>
arcq_status launch_tokens(const MoeArgs& p, int64_t m0, int64_t M) {
    const MoeWorkspace w = workspace_of(std::min<int64_t>(p.M, kMostTokens), p.top, p.K, p.I, p.N, p.E, p.perm != nullptr);
    uint8_t* at = static_cast<uint8_t*>(p.workspace);
    uint16_t* reordered = reinterpret_cast<uint16_t*>(at);
    float *h = reinterpret_cast<float*>(at + w.reordered), *partial = reinterpret_cast<float*>(at + w.reordered + w.h);
    // (a last launch of fewer tokens leaves room behind h: that of 64 tokens holds h and exponents of 4)
    uint8_t* exponents = down_few(M, p.I) ? reinterpret_cast<uint8_t*>(h + M * p.top * pitch_of(p.I)) : nullptr;
    const uint16_t* x = static_cast<const uint16_t*>(p.x) + m0 * p.ldx;
    int64_t ldx = p.ldx;
    // Up to 8192 values that have to be put in order are so by up_few_kernel itself: one token of 2048 through eight of 64 18.2 us, behind a launch that does it
    // 20.6, and 18.0 with nothing to put in order; with up to 16384 the two ways differ by 1 us to either side.
    const bool gather = p.perm && up_few(M, p.top, p.K) && M * pitch_of(p.K) <= 8 * 512 * kGathered;
    if (p.perm && !gather) {
        if (arcq_status st = launch_reorder_rows(x, M, p.K, p.ldx, p.perm, reordered, p.stream)) return st;
        x = reordered, ldx = p.K;
    }
    const int32_t* ids = p.ids + m0 * p.top;
    const int64_t most = std::min<int64_t>(p.E, M * p.top);            // experts that there can be work for
    const int tiles = (int)(p.I / 16);
    const Experts up = {p.up_codes, p.up_scales, p.up_tensor_scales, (p.K + p.S_up) / 2, (p.K + p.S_up) / B, (int)(2 * p.I)};
    const Experts down = {p.down_codes, p.down_scales, p.down_tensor_scales, (p.I + p.S_down) / 2, (p.I + p.S_down) / B, (int)p.N};
    const UpArgs u = {x, ldx, ids, p.weights + m0 * p.top, (int)M, (int)p.top, (int)p.E, (int)p.K, (int)p.I, p.activation, up, h, (int)pitch_of(p.I), exponents, tiles, gather ? p.perm : nullptr};
    if (up_few(M, p.top, p.K)) {
        const int64_t items = most * tiles;
        const int chunks = (int)((p.K + 127) / 128);
        const int kw = waves_of(chunks);
        const arcq_status st = kw == 2   ? launch_up_few<B, 2>(u, items, p.stream)
                               : kw == 4 ? launch_up_few<B, 4>(u, items, p.stream)
                                         : launch_up_few<B, 8>(u, items, p.stream);
        if (st) return st;
    } else {
        const int64_t groups = (tiles + 7) / 8;
        if (arcq_status st = M <= 16 ? launch_up_many<B, 1>(u, M * p.top * groups, p.stream) : launch_up_many<B, 2>(u, M * p.top * groups, p.stream)) return st;
    }
    DownArgs<OutT> d = {h, exponents, ids, (int)M, (int)p.top, (int)p.E, (int)p.I, (int)pitch_of(p.I), (int)p.N, down, static_cast<const OutT*>(p.residual) + (p.residual ? m0 * p.ldr : 0), p.ldr,
                        static_cast<OutT*>(p.y) + m0 * p.ldy, p.ldy, partial, (int)((p.N + 255) / 256), 1};
    if (down_few(M, p.I)) return M <= 2 ? launch_down_few<B, 2>(d, p.stream) : launch_down_few<B, 4>(d, p.stream);
    // (a last launch of fewer tokens has the runs of the first: there is room for those)
    d.splits = down_splits(std::min<int64_t>(p.M, kMostTokens), p.top, p.E, p.I, p.N);
    const int64_t items = M * p.top * d.splits * d.groups;
    if (arcq_status st = M <= 8 ? launch_down_many<B, 1>(d, items, p.stream) : launch_down_many<B, 2>(d, items, p.stream)) return st;
    const unsigned parts = (unsigned)((p.N + 255) / 256);
    hipLaunchKernelGGL((join_kernel<OutT>), dim3(parts * (unsigned)M), dim3(256), 0, p.stream, d, parts);
    return check_launch("join_kernel");
}

}  // namespace

// Enough for any number of tokens up to M: fewer may go in more runs of I and need more room for slots' results than more tokens do, so those are counted for as
// many tokens as still go in each number of runs.
size_t moe_workspace_bytes(int64_t M, int64_t top, int64_t E, int64_t K, int64_t I, int64_t N, bool reorder) {
    M = std::min<int64_t>(M, kMostTokens);
    const MoeWorkspace w = workspace_of(M, top, K, I, N, E, reorder);       // (whose other parts grow with the tokens)
    const int64_t groups = (N + 255) / 256;
    size_t partial = w.partial;
    for (int64_t runs = 2; runs <= most_runs(I); ++runs) {
        const int64_t experts = kRunItems / (groups * runs);        // that there may be work for
        partial = std::max(partial, partial_bytes(E <= experts ? M : std::min(M, experts / top), top, E, I, N));
    }
    return w.reordered + w.h + partial;
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
