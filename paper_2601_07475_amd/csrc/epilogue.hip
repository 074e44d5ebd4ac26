// The partial results of a product whose reduction dimension went in several runs, added up in index order, with what follows the sum.
// Bound by reading them (4 bytes for each run and output).
#include "epilogue.h"
#include "gemm_epilogue.h"
#include "internal.h"

#include <algorithm>

namespace arcq {

namespace {

// V outputs a thread, side by side: 4 where rows of partial results are whole pieces of 16 bytes, else 1.
template <int V, typename OutT>
__global__ __launch_bounds__(256) void splitk_epilogue_kernel(const float* __restrict__ part, int splits, int64_t split_stride, int M, int N, float alpha,
                                                              OutT* y, int64_t ldy, Epilogue<OutT> e) {
    typedef float piece_t __attribute__((ext_vector_type(V)));
    const int64_t total = (int64_t)M * (N / V);
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t m = idx / (N / V), n = V * (idx % (N / V));
        const float* at = part + m * N + n;
        float v[V], r[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            r[i] = e.residual ? (float)e.residual[m * e.ldr + n + i] : 0.0f;
            b[i] = e.bias ? (float)e.bias[n + i] : 0.0f;
        }
        piece_t sum = *reinterpret_cast<const piece_t*>(at);
        int sp = 1;
        for (; sp + 3 < splits; sp += 4) {                  // four runs' results in flight at once
            piece_t p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = *reinterpret_cast<const piece_t*>(at + (sp + k) * split_stride);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += p[k][i];
        }
        for (; sp < splits; ++sp) {
            const piece_t p = *reinterpret_cast<const piece_t*>(at + sp * split_stride);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += p[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = e.bias ? sum[i] * alpha + b[i] : sum[i] * alpha;
        activate(v, e.activation);
        if (e.residual)
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += r[i];
        if constexpr (V == 4) store4(y + m * ldy + n, v[0], v[1], v[2], v[3]);
        else store_out(y + m * ldy + n, v[0]);
    }
}

template <typename OutT>
arcq_status launch_typed(const float* partial, int splits, int M, int N, float alpha, OutT* y, int64_t ldy, const EpilogueArgs& a, hipStream_t stream) {
    const Epilogue<OutT> e = {static_cast<const _Float16*>(a.bias), static_cast<const OutT*>(a.residual), a.ldr, a.activation};
    const int64_t stride = (int64_t)M * N;
    const bool four = (N & 3) == 0;                         // (partial results are 16-byte aligned and dense)
    const int64_t work = four ? stride / 4 : stride;
    const int blocks = (int)std::min<int64_t>((work + 255) / 256, 4096);
    if (four) hipLaunchKernelGGL((splitk_epilogue_kernel<4, OutT>), dim3(blocks), dim3(256), 0, stream, partial, splits, stride, M, N, alpha, y, ldy, e);
    else hipLaunchKernelGGL((splitk_epilogue_kernel<1, OutT>), dim3(blocks), dim3(256), 0, stream, partial, splits, stride, M, N, alpha, y, ldy, e);
    return check_launch("splitk_epilogue_kernel");
}

}  // namespace

arcq_status launch_splitk_epilogue(const float* partial, int splits, int M, int N, float alpha, void* y, int y_dtype, int64_t ldy, const EpilogueArgs& e,
                                   hipStream_t stream) {
    return y_dtype == ARCQ_DTYPE_F16 ? launch_typed(partial, splits, M, N, alpha, static_cast<_Float16*>(y), ldy, e, stream)
                                     : launch_typed(partial, splits, M, N, alpha, static_cast<float*>(y), ldy, e, stream);
}

}  // namespace arcq
