// Types shared by the MX4 GEMM kernels (included by gemm_mx4.hip only).
#pragma once

#include "gemm_dl.h"
#include "mx4.h"

namespace occ {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// C (M x N) = A (M x K) B (N x K)^T in the layout of mx4.h.
struct Mx4Operands {
  const uint8_t *A, *As, *B, *Bs;
  void *C;
  int M, N;
  uint32_t pitch;  // bytes of a row of codes, and of a row of scale tiles
  int steps256;    // ceil(K / 256)
  int steps512;    // ceil(K / 512) = pitch / 256
};

// One 16x16x128 MFMA of E2M1 operands, 16 bytes a lane: lane l feeds row l % 16 and
// columns 32 (l / 16) .. + 31 of the step, one block of the format; byte Q of its
// scale word is that block's scale.
template <int Q>
__device__ __forceinline__ f32x4 mfma_mx4(u32x4 a, u32x4 b, f32x4 c, int a_scale, int b_scale) {
  constexpr int kE2M1 = 4;
  const i32x8 a8 = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 b8 = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, kE2M1, kE2M1, Q, a_scale, Q, b_scale);
}

// Two neighbouring 16x16 blocks of C^T (columns n0 .. n0 + 31 of rows mb .. mb + 15):
// lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of each.
__device__ __forceinline__ void store_mx4_pair(uint16_t *C, int M, int N, int mb, int em, int n0, int lane, f32x4 p,
                                               f32x4 q) {
  u32x4 v;  // swapping odd rows of lanes of one block with even rows of the other: 8 columns a lane
#pragma unroll
  for (int d = 0; d < 2; ++d) {
    const auto s = __builtin_amdgcn_permlane16_swap(pack_bf16(p[2 * d], p[2 * d + 1]),
                                                    pack_bf16(q[2 * d], q[2 * d + 1]), false, false);
    v[d] = s[0];
    v[2 + d] = s[1];
  }
  const int n = n0 + ((lane >> 4) & 1) * 16 + (lane >> 5) * 8;
  if (mb + em < M) store_c_ragged(C + (size_t)(mb + em) * N + n, v, N - n, false);
}
__device__ __forceinline__ void store_mx4_pair(float *C, int M, int N, int mb, int em, int n0, int lane, f32x4 p,
                                               f32x4 q) {
  typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
  if (mb + em >= M) return;
  const int n = n0 + (lane >> 4) * 4;
  float *row = C + (size_t)(mb + em) * N;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const f32x4 v = b ? q : p;
    const int at = n + 16 * b;
    if (at + 4 <= N) {
      __builtin_nontemporal_store(v, reinterpret_cast<f32x4_a4 *>(row + at));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < N) row[at + e] = v[e];
    }
  }
}

}  // namespace
}  // namespace occ
