// What a product does with its sums behind them: y = act(sum + bias[n]) + residual[m, n], in fp32, rounded once to y's type.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/arcq.h"
#include "gemm_epilogue.h"

namespace arcq {

// Products that end with their sums.
struct NoEpilogue {};

// bias: fp16 [N] or null; residual: [M, N] of y's type, pitch ldr, or null (it may be y itself: an element is read by the lane that writes it)
template <typename OutT>
struct Epilogue {
    const _Float16* bias;
    const OutT* residual;
    int64_t ldr;
    int activation;
};

// y of a kernel.  Where there may be a residual that is y, its memory is read through another pointer than it is written through.
template <typename OutT, typename Ep>
using OutputOf = std::conditional_t<std::is_same<Ep, NoEpilogue>::value, OutT* __restrict__, OutT*>;

constexpr float kLog2e = 1.44269504088896340736f;

// v / (1 + exp(-t)): the exponential by v_exp_f32, the quotient by v_rcp_f32, each within one unit of fp32's last place.  Where the exponential
// overflows the quotient is 0, as it is in the limit.
__device__ __forceinline__ float times_sigmoid(float v, float t) {
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * t));
}

// v Phi(v) = v erfc(-v / sqrt(2)) / 2, within 20 units of 2^-24 of its value on either side (11.6 at most in an evaluation of these steps in fp32 over 500000 arguments with every
// error of v_rcp_f32 and v_exp_f32).  With z = |v| / sqrt(2), exp(z z) erfc(z) is 2 t times a polynomial of degree eight in t = 1 / (1 + 3 z / 8), fitted to it over 0 <= z <= 10.4
// by least squares whose weights are raised where the relative error is largest (Lawson's method): 2^-26 of it at most.  exp(-z z) is 2^-(c v v): what rounding leaves
// of the square and of its product with c is put back on the power, or it would be wrong by c v v units.  24 instructions; a polynomial of degree five without
// that (14) is right to 1.5e-7 but not in the tail, where little is left of v (4.7e-4 of it at -4).  333 x 27648 over K = 5120 in fp16 98.5 -> 103.5 us for it.
__device__ __forceinline__ float gelu_erf(float v) {
    const float a = __builtin_fminf(__builtin_fabsf(v), 16.0f);         // (nothing of fp32 is left of the tail there)
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.375f * 0.70710678118654752440f, a, 1.0f));
    float p = __builtin_fmaf(3.055110015e-02f, t, -1.426360607e-01f);
    p = __builtin_fmaf(p, t, 2.141363919e-01f);
    p = __builtin_fmaf(p, t, -1.124154404e-01f);
    p = __builtin_fmaf(p, t, 1.353237629e-01f);
    p = __builtin_fmaf(p, t, 6.139074266e-02f);
    p = __builtin_fmaf(p, t, 1.024973169e-01f);
    p = __builtin_fmaf(p, t, 1.053467095e-01f);
    p = __builtin_fmaf(p, t, 1.058054715e-01f);
    constexpr float C = 0.5f * kLog2e, C_REST = (float)(0.5 * 1.44269504088896340736 - (double)C);
    const float square = a * a, x = square * C;
    const float rest = __builtin_fmaf(__builtin_fmaf(a, a, -square), C, __builtin_fmaf(square, C_REST, __builtin_fmaf(square, C, -x)));
    const float e = __builtin_amdgcn_exp2f(-x);
    const float tail = a * (p * t * __builtin_fmaf(e, -0.69314718055994530942f * rest, e));      // |v| Phi(-|v|)
    return v > 0.0f ? v - tail : v < 0.0f ? -tail : v;
}

// v Phi(v) by 0.5 v (1 + tanh u) = v / (1 + exp(-2 u)), u = sqrt(2 / pi) (v + 0.044715 v^3)
__device__ __forceinline__ float gelu_tanh(float v) {
    const float u2 = 1.59576912160573071176f * __builtin_fmaf(0.044715f * v * v, v, v);
    return times_sigmoid(v, u2);
}

// The same activation for N values; which one is uniform over a launch.
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int activation) {
    if (activation == ARCQ_ACT_NONE) return;
    if (activation == ARCQ_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = times_sigmoid(v[i], v[i]);
    } else if (activation == ARCQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    } else if (activation == ARCQ_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu_erf(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = gelu_tanh(v[i]);
    }
}

// One output.
template <typename OutT>
__device__ __forceinline__ float finish(const NoEpilogue&, float sum, int64_t, int64_t) { return sum; }
template <typename OutT>
__device__ __forceinline__ float finish(const Epilogue<OutT>& e, float sum, int64_t m, int64_t n) {
    float v[1] = {sum};
    const float r = e.residual ? (float)e.residual[m * e.ldr + n] : 0.0f;
    if (e.bias) v[0] += (float)e.bias[n];
    activate(v, e.activation);
    return e.residual ? v[0] + r : v[0];
}

// The same in two steps: what it reads, early, and the rest.
template <typename Ep>
struct Operands {                                   // of NoEpilogue
    __device__ __forceinline__ void ask(const Ep&, int64_t, int64_t) {}
    __device__ __forceinline__ float finish(const Ep&, float sum) const { return sum; }
};
template <typename OutT>
struct Operands<Epilogue<OutT>> {
    _Float16 bias = (_Float16)0.0f;
    OutT residual = (OutT)0.0f;
    __device__ __forceinline__ void ask(const Epilogue<OutT>& e, int64_t m, int64_t n) {
        if (e.bias) bias = e.bias[n];
        if (e.residual) residual = e.residual[m * e.ldr + n];
    }
    __device__ __forceinline__ float finish(const Epilogue<OutT>& e, float sum) const {
        float v[1] = {e.bias ? sum + (float)bias : sum};
        activate(v, e.activation);
        return e.residual ? v[0] + (float)residual : v[0];
    }
};

// A wave's tile of 32 WM x 32 WN sums (accumulator layout as in store_tile_swapped), a fragment row of 32 at a time through the wave's region of LDS in
// fp32: the bias on the way in, where a lane holds four columns side by side; the activation in place, in a loop whose body is there four times (unrolled over
// the accumulator registers, four activations would fill the instruction cache); the residual on the way out, where a wave's loads and stores are
// whole lines.  A fragment row's residual is asked for before the one before it is worked on.
// lds_wave: epilogue_lds_bytes(WN) bytes, as in store_fragment_rows_f16_via_lds.
// Measured: 4096 x 8192 over K = 28672 with a residual in fp16 1.20 to 1.26 ms, the product alone 1.21 to 1.24 (1.28 where every row asked for its own and looked for the edge
// value by value); 333 x 27648 over 5120 with SiLU 93 us, alone 90 to 97; 777 x 6147 over 4352 with everything, fp32, 66 us, alone 54 (one
// round of tiles, all at their ends at the same time).
template <int WM, int WN, typename OutT, bool INSIDE>
struct TileEnd {
    typedef float float4v __attribute__((ext_vector_type(4)));
    static constexpr int V = 16 / (int)sizeof(OutT);                    // a lane's 16 bytes of y
    typedef OutT piece_t __attribute__((ext_vector_type(V), aligned(sizeof(OutT))));
    static constexpr int PITCH = 128 * WN + 16;                         // (the padding spreads the rows over the banks)
    static constexpr int LPR = 32 * WN / V, RPI = 64 / LPR, PASSES = 32 / RPI;      // lanes of a row; rows of a store instruction
    static_assert(32 * PITCH <= epilogue_lds_bytes(WN), "a fragment row in fp32 fits the region");

    const float16v (&acc)[WM][WN];
    uint8_t* lds_wave;
    int m0, n0, lane, M, N;
    OutT* y;
    int64_t ldy;
    const Epilogue<OutT>& e;

    __device__ __forceinline__ void ask(int i, piece_t (&res)[PASSES]) const {
        if (!e.residual) return;
        const int row0 = lane / LPR, n = n0 + V * (lane % LPR);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int m = m0 + 32 * i + p * RPI + row0;
            const OutT* at = e.residual + (int64_t)m * e.ldr + n;
            if (INSIDE || (m < M && n + V <= N)) {
                res[p] = *reinterpret_cast<const piece_t*>(at);
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    res[p][k] = (OutT)0.0f;
                    if (m < M && n + k < N) res[p][k] = at[k];
                }
            }
        }
    }
    template <int I>
    __device__ __forceinline__ void finish(const float (&bias)[WN][16], const piece_t (&res)[PASSES]) const {
        const int r = lane & 31, h = lane >> 5, row0 = lane / LPR, n = n0 + V * (lane % LPR);
        uint8_t* own = lds_wave + r * PITCH + 16 * h;
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4v*>(own + 128 * j + 32 * g) = float4v{acc[I][j][4 * g] + bias[j][4 * g], acc[I][j][4 * g + 1] + bias[j][4 * g + 1],
                                                                              acc[I][j][4 * g + 2] + bias[j][4 * g + 2], acc[I][j][4 * g + 3] + bias[j][4 * g + 3]};
        if (e.activation != ARCQ_ACT_NONE) {
#pragma unroll 1
            for (int k = 0; k < 4 * WN; k += 4) {
                float v[16];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4v t = *reinterpret_cast<const float4v*>(own + 32 * (k + g));
                    v[4 * g] = t[0], v[4 * g + 1] = t[1], v[4 * g + 2] = t[2], v[4 * g + 3] = t[3];
                }
                activate(v, e.activation);
#pragma unroll
                for (int g = 0; g < 4; ++g) *reinterpret_cast<float4v*>(own + 32 * (k + g)) = float4v{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
            }
        }
        // the reads below take what other lanes of this wave wrote: LDS operations of a wave complete in order
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int m = m0 + 32 * I + p * RPI + row0;
            const uint8_t* from = lds_wave + (p * RPI + row0) * PITCH + 4 * V * (lane % LPR);
            piece_t out;
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const float4v t = *reinterpret_cast<const float4v*>(from + 4 * k);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[k + i] = (OutT)(e.residual ? t[i] + (float)res[p][k + i] : t[i]);
            }
            if (!INSIDE && m >= M) continue;
            OutT* dst = y + (int64_t)m * ldy + n;
            if (INSIDE || n + V <= N) {
                *reinterpret_cast<piece_t*>(dst) = out;
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (n + k < N) dst[k] = out[k];
            }
        }
        // the next fragment row reuses the region
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    __device__ __forceinline__ void run() const {
        float bias[WN][16];                     // of the lane's columns, in the accumulators' order
#pragma unroll
        for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = n0 + 32 * j + 8 * g + 4 * (lane >> 5);
#pragma unroll
                for (int k = 0; k < 4; ++k) bias[j][4 * g + k] = 0.0f;
                if (!e.bias) continue;
                if (INSIDE) {
                    const half4_a2 v = *reinterpret_cast<const half4_a2*>(e.bias + n);
#pragma unroll
                    for (int k = 0; k < 4; ++k) bias[j][4 * g + k] = (float)v[k];
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (n + k < N) bias[j][4 * g + k] = (float)e.bias[n + k];
                }
            }
        piece_t even[PASSES], odd[PASSES];
        ask(0, even);
        if constexpr (WM > 1) ask(1, odd);
        finish<0>(bias, even);
        if constexpr (WM > 2) ask(2, even);
        if constexpr (WM > 1) finish<1>(bias, odd);
        if constexpr (WM > 3) ask(3, odd);
        if constexpr (WM > 2) finish<2>(bias, even);
        if constexpr (WM > 3) finish<3>(bias, odd);
        static_assert(WM <= 4, "up to four fragment rows");
    }
};

template <int WM, int WN, typename OutT>
__device__ __forceinline__ void finish_tile(const float16v (&acc)[WM][WN], uint8_t* lds_wave, int m0, int n0, int lane, int M, int N, OutT* y, int64_t ldy,
                                            const Epilogue<OutT>& e) {
    if (m0 + 32 * WM <= M && n0 + 32 * WN <= N) TileEnd<WM, WN, OutT, true>{acc, lds_wave, m0, n0, lane, M, N, y, ldy, e}.run();
    else TileEnd<WM, WN, OutT, false>{acc, lds_wave, m0, n0, lane, M, N, y, ldy, e}.run();
}

}  // namespace arcq
