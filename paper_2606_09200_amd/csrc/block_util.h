// Loads, stores and sums shared by the block operators' kernels.
#pragma once

#include "gemm_common.h"

namespace occ {
namespace {

typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any element
typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));

// By value: a bit cast of a vector's element itself would read its first.
__device__ __forceinline__ float as_float(uint32_t w) { return __builtin_bit_cast(float, w); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }

__device__ __forceinline__ float value(uint16_t h) { return as_float((uint32_t)h << 16); }
__device__ __forceinline__ float value(float f) { return f; }

// 8 consecutive values of a row as they are stored (bf16: 4 words, binary32: 8); the first
// `left` of them exist, the others are zero.  Rows start at any element.
// Element `at` of a row: a 32-bit byte offset from a uniform base costs one register, a pointer per
// lane two.
template <class E>
__device__ __forceinline__ E *element(E *row, uint32_t at) {
  typedef std::conditional_t<std::is_const<E>::value, const char, char> Byte;
  return reinterpret_cast<E *>(reinterpret_cast<Byte *>(row) + at * (uint32_t)sizeof(E));
}

template <class E>
struct Raw8;
template <>
struct Raw8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t *p, int left) {
    w = u32x4{0u, 0u, 0u, 0u};
    if (left >= 8) {
      w = *reinterpret_cast<const u32x4_e2 *>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t lo = 0u, hi = 0u;
        if (2 * i < left) lo = p[2 * i];
        if (2 * i + 1 < left) hi = p[2 * i + 1];
        w[i] = lo | hi << 16;
      }
    }
  }
  __device__ __forceinline__ float at(int e) const { return e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }
};
template <>
struct Raw8<float> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const float *p, int left) {
    a = b = u32x4{0u, 0u, 0u, 0u};
    if (left >= 8) {
      a = *reinterpret_cast<const u32x4_e4 *>(p);
      b = *reinterpret_cast<const u32x4_e4 *>(p + 4);
    } else {
      const uint32_t *w = reinterpret_cast<const uint32_t *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < left) a[i] = w[i];
        if (4 + i < left) b[i] = w[4 + i];
      }
    }
  }
  __device__ __forceinline__ float at(int e) const { return e < 4 ? as_float(a[e]) : as_float(b[e - 4]); }
};

// The same as binary32 values.
template <class E>
__device__ __forceinline__ void load8(const E *p, int left, float (&v)[8]) {
  Raw8<E> r;
  r.load(p, left);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r.at(e);
}

// 8 consecutive values of a row, rounded to the row's type; the first `left` of them exist.
// Non-temporal: outputs as large as these are not read again before they leave the L2.
__device__ __forceinline__ void store8(uint16_t *p, int left, const float (&v)[8]) {
  if (left >= 8) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_e2 *>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = to_bf16(v[i]);
  }
}
__device__ __forceinline__ void store8(float *p, int left, const float (&v)[8]) {
  if (left >= 8) {
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __builtin_bit_cast(uint32_t, v[i]);
      b[i] = __builtin_bit_cast(uint32_t, v[4 + i]);
    }
    __builtin_nontemporal_store(a, reinterpret_cast<u32x4_e4 *>(p));
    __builtin_nontemporal_store(b, reinterpret_cast<u32x4_e4 *>(p + 4));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = v[i];
  }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return as_float((uint32_t)__builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}

// Sum over a wave's 64 lanes, the same bits in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  v = v + dpp<0xB1>(v);   // lane ^ 1
  v = v + dpp<0x4E>(v);   // lane ^ 2
  v = v + dpp<0x141>(v);  // the other quad of 8 lanes
  v = v + dpp<0x140>(v);  // the other half of 16 lanes
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  v = as_float(s[0]) + as_float(s[1]);
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  const auto t = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return as_float(t[0]) + as_float(t[1]);
}

}  // namespace
}  // namespace occ
