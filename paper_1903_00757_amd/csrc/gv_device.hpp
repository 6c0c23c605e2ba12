// Device functions shared by the kernels of training (gv_kernels.hip) and of rows (gv_rows.hip, gv_scores.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gv {
namespace {

// ---------------------------------------------------------------------------
// Philox4x32-10 (Salmon et al., SC'11): ten rounds of two 32x32->64 multiplies
// and a word permutation; the key advances by the Weyl constants between rounds.  kJoined: the two exclusive ors of a word are
// one instruction; the kernels of training leave them to the compiler.
template <bool kJoined = false>
__device__ __forceinline__ uint4 philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                               uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        if constexpr (kJoined) {  // 0x96: the truth table of a ^ b ^ c
            c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(p1 >> 32), c1, k0, 0x96);
            c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(p0 >> 32), c3, k1, 0x96);
        } else {
            c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
            c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        }
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// A DPP move: lane l takes x of the lane that kCtrl names, 0 in the rows that are masked out.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp_take(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, kRowMask, 0xF, false));
}

}  // namespace
}  // namespace gv
