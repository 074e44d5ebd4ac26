// 4 x 4 transposes across the four groups of 16 lanes of a wave, shared by the weight-streaming kernels: lane (i, q), q = lane / 16, gets
// element q of what lanes (i, 0) to (i, 3) held.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace arcq {

typedef unsigned uint2v __attribute__((ext_vector_type(2)));

// Of the bytes of a word.  sel_half: 0x05040100 for q < 2, else 0x07060302; sel_byte: 0x06020400 for even q, else 0x07030501.
__device__ __forceinline__ uint32_t transpose_scale_bytes(uint32_t s, uint32_t sel_half, uint32_t sel_byte) {
    const uint2v x = __builtin_amdgcn_permlane32_swap(s, s, false, false);     // (q, q ^ 2): own and partner word
    const uint32_t pair = __builtin_amdgcn_perm(x[1], x[0], sel_half);         // bytes {0,1} or {2,3} of chunks (q & 1), (q & 1) + 2
    const uint2v t = __builtin_amdgcn_permlane16_swap(pair, pair, false, false);   // (q, q ^ 1)
    return __builtin_amdgcn_perm(t[1], t[0], sel_byte);                        // byte q of chunks 0, 1, 2, 3
}
__device__ __forceinline__ uint32_t half_selector(int q) { return q < 2 ? 0x05040100u : 0x07060302u; }
__device__ __forceinline__ uint32_t byte_selector(int q) { return (q & 1) ? 0x07030501u : 0x06020400u; }

// Of the words of 16 bytes.
__device__ __forceinline__ void transpose_words(uint4& w) {
    const uint2v a = __builtin_amdgcn_permlane32_swap(w.x, w.z, false, false), b = __builtin_amdgcn_permlane32_swap(w.y, w.w, false, false);
    const uint2v c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w = make_uint4(c[0], c[1], d[0], d[1]);
}

}  // namespace arcq
