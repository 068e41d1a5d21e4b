// Division of numbers below 2^31 by one that a launch fixes.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define OCC_DIVIDE __host__ __device__ __forceinline__
#else
#define OCC_DIVIDE inline
#endif

namespace occ {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31.  With 2^(s-1) < d <= 2^s and mul = floor(2^32 (2^s - d) / d) + 1, the
// quotient is (mulhi(n, mul) + n) >> s (Granlund and Montgomery 1994), and the sum stays below 2^32.
struct Divider {
  uint32_t mul;
  int shift;
  Divider() = default;
  explicit Divider(int d) : mul(0), shift(0) {
    while ((1u << shift) < (uint32_t)d) ++shift;
    mul = (uint32_t)(((uint64_t)((1u << shift) - (uint32_t)d) << 32) / (uint32_t)d + 1);
  }
  OCC_DIVIDE int operator()(int n) const {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t high = __umulhi((uint32_t)n, mul);
#else
    const uint32_t high = (uint32_t)(((uint64_t)(uint32_t)n * mul) >> 32);
#endif
    return (int)((high + (uint32_t)n) >> shift);
  }
};

}  // namespace occ
