// What the decoding operators (include/atk_decode.h) share.
#pragma once

#include <algorithm>

#include "atk_common.h"
#include "../../include/atk_decode.h"

namespace atk {

// Quotients of 31-bit numbers by a number that the host knows: q = (hi(M * n) + n) >> s with s = ceil(log2 d), M = floor(2^32 (2^s - d) / d) + 1.
struct FastDiv {
    uint32_t d, mul, shift;
    void set(uint32_t divisor) {
        d = divisor;
        shift = 0;
        while (shift < 31 && (1u << shift) < d) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
#ifdef __HIPCC__
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
    __device__ __forceinline__ int mod(int n) const { return n - div(n) * (int)d; }
#endif
};

// A launch has fewer than 2^32 threads; past that HIP refuses it.
constexpr bool launches(int64_t workgroups, int threads) { return workgroups < (INT64_C(1) << 32) / threads; }

int set_hip_error(hipError_t e);  // ATK_ERR_HIP, with e for atk_last_hip_error()

}  // namespace atk
