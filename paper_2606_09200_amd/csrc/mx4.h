// The MX4 format (include/occ.h) on the device: layout and conversions.
#pragma once

#include "occ_internal.h"

namespace occ {
namespace {

constexpr int kMx4Tile = 512;  // columns of a scale tile; rows are padded to a multiple

// Byte of a 16 x 512 scale tile that holds row r of the tile's (r < 16) and
// block b (b < 16) of its 16 blocks of 32 columns.
__device__ __forceinline__ int mx4_scale_byte(int r, int b) { return ((b & 3) * 16 + r) * 4 + (b >> 2); }

// Scale byte of a block whose largest |x| has the binary32 bits `top`:
// floor(log2) - 2 + 127.  Zeros and subnormals (exponent field 0) and everything
// below 2^-125 get 0 (2^-127); infinities and NaN, whose field is 255, get 255.
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top) {
  const int f = (int)(top >> 23);
  return f == 255 ? 255u : (uint32_t)max(0, f - 2);
}

// 2^(s - 127) as binary32 (s = 0 is a subnormal); NaN for s = 255.
__device__ __forceinline__ float mx4_scale_value(uint32_t s) {
  const uint32_t bits = s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23;
  return __builtin_bit_cast(float, bits);
}

}  // namespace
}  // namespace occ
