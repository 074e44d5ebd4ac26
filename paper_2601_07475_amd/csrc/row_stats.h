// Mean of squares of a row with an EXACT sum, shared by the kernels with RMSNorm in front of a quantizer.
//
// fp16 values times 2^24 are integers below 2^40; split as a 2^20 + b with a, b < 2^20, the squares add up as three integer sums,
// and only the joined sum is rounded, once, to fp64.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace arcq {

// Sum of v over each row of 16 lanes, in every lane of the row (data-parallel-primitive moves within
// quads, half rows and rows).
template <int CTRL>
__device__ __forceinline__ double dpp_move(double v) {
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true);
    return __hiloint2double(hi, lo);
}
__device__ __forceinline__ double row16_sum(double v) {
    v += dpp_move<0xB1>(v);     // quad_perm [1,0,3,2]
    v += dpp_move<0x4E>(v);     // quad_perm [2,3,0,1]
    v += dpp_move<0x141>(v);    // row_half_mirror
    v += dpp_move<0x140>(v);    // row_mirror
    return v;
}

// s_aa 2^40 + s_ab 2^21 + s_bb (< 2^97, the sum of squares in units of 2^-48), rounded once: six exact doubles are added
// without error into (hi, lo); hi + lo then rounds the exact integer.
__device__ __forceinline__ double join_exact_sums(uint64_t s_aa, uint64_t s_ab, uint64_t s_bb) {
    const double term[6] = {(double)(uint32_t)(s_aa >> 32) * 0x1p72, (double)(uint32_t)s_aa * 0x1p40,
                            (double)(uint32_t)(s_ab >> 32) * 0x1p53, (double)(uint32_t)s_ab * 0x1p21,
                            (double)(uint32_t)(s_bb >> 32) * 0x1p32, (double)(uint32_t)s_bb};
    double hi = term[0], lo = 0.0;
#pragma unroll
    for (int k = 1; k < 6; ++k) {
        const double sum = hi + term[k];
        const double bb = sum - hi;
        const double err = (hi - (sum - bb)) + (term[k] - bb);   // hi + term = sum + err exactly
        hi = sum;
        lo += err;           // integers below 2^53: exact
    }
    return (hi + lo) * 0x1p-48;
}

}  // namespace arcq
