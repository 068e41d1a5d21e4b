// Loads, stores and sums shared by the block operators' kernels.
#pragma once

#include "gemm_common.h"

namespace occ {
namespace {

typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));  // 16 bytes at any element
typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x2_e4 __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_e2 __attribute__((aligned(2)));

// By value: a bit cast of a vector's element itself would read its first.
__device__ __forceinline__ float as_float(uint32_t w) { return __builtin_bit_cast(float, w); }
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }

__device__ __forceinline__ float value(uint16_t h) { return as_float((uint32_t)h << 16); }
__device__ __forceinline__ float value(float f) { return f; }

// Element `at` of a row: a 32-bit byte offset from a uniform base costs one register, a pointer per
// lane two.
template <class E>
__device__ __forceinline__ E *element(E *row, uint32_t at) {
  typedef std::conditional_t<std::is_const<E>::value, const char, char> Byte;
  return reinterpret_cast<E *>(reinterpret_cast<Byte *>(row) + at * (uint32_t)sizeof(E));
}

// 8 consecutive values of a row as they are stored (bf16: 4 words, binary32: 8), zeros where they do
// not exist.  Rows start at any element.  load: all of them or none; load_part: the first
// `left`, the end of a row of `cols` values: the lane there takes the row's last 8 and shifts
// out those it does not own (one load and a few selects).
template <class E>
struct Raw8;
template <>
struct Raw8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t *p, bool in) {
    w = u32x4{0u, 0u, 0u, 0u};
    if (in) w = *reinterpret_cast<const u32x4_e2 *>(p);
  }
  __device__ __forceinline__ void load_rest(const uint16_t *p, int cols) {  // see store_rest
    if (cols & 4) {
      const u32x2_e2 v = *reinterpret_cast<const u32x2_e2 *>(p);
      w[0] = v[0], w[1] = v[1];
      p += 4;
    }
    if (cols & 2) {
      w[2] = *reinterpret_cast<const u32_e2 *>(p);
      p += 2;
    }
    if (cols & 1) w[3] = *p;
  }
  __device__ __forceinline__ void load_part(const uint16_t *p, int left, int cols) {
    w = u32x4{0u, 0u, 0u, 0u};
    if (cols >= 8) {
      const int drop = 8 - (cols & 7);  // the same for every row
      const bool part = left < 8;
      if (left > 0) w = *reinterpret_cast<const u32x4_e2 *>(part ? p - drop : p);
      const bool d4 = part && (drop & 4), d2 = part && (drop & 2), d1 = part && (drop & 1);
      w[0] = d4 ? w[2] : w[0];
      w[1] = d4 ? w[3] : w[1];
      w[2] = d4 ? 0u : w[2];
      w[3] = d4 ? 0u : w[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = d2 ? (i < 3 ? w[i + 1] : 0u) : w[i];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = d1 ? __builtin_amdgcn_alignbit(i < 3 ? w[i + 1] : 0u, w[i], 16) : w[i];
    } else if (left > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = p[min(2 * i, left - 1)], hi = p[min(2 * i + 1, left - 1)];
        w[i] = (2 * i < left ? lo : 0u) | (2 * i + 1 < left ? hi << 16 : 0u);
      }
    }
  }
  __device__ __forceinline__ float at(int e) const { return e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }
  // What was computed from the words so far is computed again, not kept in registers.
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(w)); }
};
template <>
struct Raw8<float> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const float *p, bool in) {
    a = b = u32x4{0u, 0u, 0u, 0u};
    if (in) {
      a = *reinterpret_cast<const u32x4_e4 *>(p);
      b = *reinterpret_cast<const u32x4_e4 *>(p + 4);
    }
  }
  __device__ __forceinline__ void load_rest(const float *p, int cols) {
    if (cols & 4) {
      a = *reinterpret_cast<const u32x4_e4 *>(p);
      p += 4;
    }
    if (cols & 2) {
      const u32x2_e4 v = *reinterpret_cast<const u32x2_e4 *>(p);
      b[0] = v[0], b[1] = v[1];
      p += 2;
    }
    if (cols & 1) b[2] = *reinterpret_cast<const uint32_t *>(p);
  }
  __device__ __forceinline__ void load_part(const float *p, int left, int cols) {
    a = b = u32x4{0u, 0u, 0u, 0u};
    if (cols >= 8) {
      const int drop = 8 - (cols & 7);
      const bool part = left < 8;
      if (left > 0) {
        const float *q = part ? p - drop : p;
        a = *reinterpret_cast<const u32x4_e4 *>(q);
        b = *reinterpret_cast<const u32x4_e4 *>(q + 4);
      }
      const u32x4 none = {0u, 0u, 0u, 0u};
      const bool d4 = part && (drop & 4), d2 = part && (drop & 2), d1 = part && (drop & 1);
      a = d4 ? b : a;
      b = d4 ? none : b;
      a = d2 ? u32x4{a[2], a[3], b[0], b[1]} : a;
      b = d2 ? u32x4{b[2], b[3], 0u, 0u} : b;
      a = d1 ? u32x4{a[1], a[2], a[3], b[0]} : a;
      b = d1 ? u32x4{b[1], b[2], b[3], 0u} : b;
    } else if (left > 0) {
      const uint32_t *w = reinterpret_cast<const uint32_t *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = w[min(i, left - 1)], hi = w[min(4 + i, left - 1)];
        a[i] = i < left ? lo : 0u;
        b[i] = 4 + i < left ? hi : 0u;
      }
    }
  }
  __device__ __forceinline__ float at(int e) const { return e < 4 ? as_float(a[e]) : as_float(b[e - 4]); }
  __device__ __forceinline__ void forget() { asm volatile("" : "+v"(a), "+v"(b)); }
};

// 8 consecutive values of a row, rounded to the row's type, where they exist.
// NT: non-temporal.
template <bool NT = true>
__device__ __forceinline__ void store8(uint16_t *p, bool in, const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  if (NT) {
    if (in) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_e2 *>(p));
  } else {
    if (in) *reinterpret_cast<u32x4_e2 *>(p) = w;
  }
}
template <bool NT = true>
__device__ __forceinline__ void store8(float *p, bool in, const float (&v)[8]) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __builtin_bit_cast(uint32_t, v[i]);
    b[i] = __builtin_bit_cast(uint32_t, v[4 + i]);
  }
  if (in) {
    if (NT) {
      __builtin_nontemporal_store(a, reinterpret_cast<u32x4_e4 *>(p));
      __builtin_nontemporal_store(b, reinterpret_cast<u32x4_e4 *>(p + 4));
    } else {
      *reinterpret_cast<u32x4_e4 *>(p) = a;
      *reinterpret_cast<u32x4_e4 *>(p + 4) = b;
    }
  }
}

// The end of a row of `cols` values, cols % 8 of them, taken by fours, twos and ones: as far as there
// are any, elements 0 to 3, then 4 and 5, then 6.
template <class E>
__device__ __forceinline__ void store_rest(E *p, int cols, const float (&v)[8]) {
  auto put = [&](float x) {
    if constexpr (sizeof(E) == 2) *p++ = to_bf16(x);
    else *p++ = x;
  };
  if (cols & 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) put(v[i]);
  }
  if (cols & 2) {
    put(v[4]);
    put(v[5]);
  }
  if (cols & 1) put(v[6]);
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
