// Skinny (M <= 16) MX4 GEMM (included by gemm_mx4.hip only).
#pragma once

#include "gemm_mx4_common.h"

namespace occ {
namespace {

// ---------------------------------------------------------------------------
// M <= 16 (decode-like, bound by reading B once).  A unit is UT blocks of 16
// columns of C (16 rows of B) over the whole K; KW waves of a workgroup take its
// 512-wide k-steps in turn, so that together they read KW * 256 contiguous bytes of
// every row, and 8 / KW units share a workgroup.  A wave has the codes and scales
// of U k-steps in flight straight to registers; a lane's 16 bytes are one block of
// 32 columns, its word of the scale tile serves all four MFMAs of the k-step.  The
// KW partial sums are added in wave order through LDS: the result does not depend
// on timing.  Rows of A past M and rows of B past N lie beyond their descriptors
// and read as zero.
template <int KW, int UT, class OUT, bool NT>
__global__ __launch_bounds__(512) void gemm_mx4_skinny_kernel(Mx4Operands o, int units) {
  constexpr int U = 2, WPU = 8 / KW;
  __shared__ f32x4 partial[8][UT][64];
  extern __shared__ __align__(16) unsigned char pad_lds[];  // occupancy pad only
  (void)pad_lds;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave % KW;
  const int unit = blockIdx.x * WPU + wave / KW;
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t P = o.pitch;
  const int n0 = unit * 16 * UT;
  const int nk = unit < units ? o.steps512 : 0;
  const int rows = max(0, min(16 * UT, o.N - n0));
  const size_t first = unit < units ? (size_t)n0 : 0;
  const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.B) + first * P, 0,
                                                    (int)((uint32_t)rows * P), 0x00020000);
  const auto rbs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.Bs) + (first >> 4) * P, 0,
                                                     (int)((uint32_t)((rows + 15) >> 4) * P), 0x00020000);
  const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.A), 0, (int)((uint32_t)o.M * P), 0x00020000);
  const auto ras = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.As), 0, (int)P, 0x00020000);
  constexpr int kPolicy = NT ? 2 : 0;
  const uint32_t off = (uint32_t)l16 * P + (uint32_t)g * 16u;

  f32x4 acc[UT];
#pragma unroll
  for (int i = 0; i < UT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = kw; k < nk; k += KW * U) {
    u32x4 b[U][UT][4], a[U][4];
    int bs[U][UT], as[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kk = k + u * KW;
      const uint32_t k0 = kk < nk ? (uint32_t)kk * 256u : 0x80000000u;  // past the end: nothing is read
#pragma unroll
      for (int i = 0; i < UT; ++i) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
          b[u][i][s] = __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(off + (uint32_t)(i * 16) * P + s * 64u + k0), 0, kPolicy);
        bs[u][i] = (int)__builtin_amdgcn_raw_buffer_load_b32(rbs, (int)((uint32_t)i * P + lane * 4u + k0), 0, kPolicy);
      }
#pragma unroll
      for (int s = 0; s < 4; ++s) a[u][s] = __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(off + s * 64u + k0), 0, 0);
      as[u] = (int)__builtin_amdgcn_raw_buffer_load_b32(ras, (int)(lane * 4u + k0), 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < UT; ++i) {
        acc[i] = mfma_mx4<0>(b[u][i][0], a[u][0], acc[i], bs[u][i], as[u]);
        acc[i] = mfma_mx4<1>(b[u][i][1], a[u][1], acc[i], bs[u][i], as[u]);
        acc[i] = mfma_mx4<2>(b[u][i][2], a[u][2], acc[i], bs[u][i], as[u]);
        acc[i] = mfma_mx4<3>(b[u][i][3], a[u][3], acc[i], bs[u][i], as[u]);
      }
  }
  if constexpr (KW > 1) {
    if (kw > 0) {
#pragma unroll
      for (int i = 0; i < UT; ++i) partial[wave][i][lane] = acc[i];
    }
    __syncthreads();
    if (kw > 0) return;
#pragma unroll
    for (int i = 0; i < UT; ++i)
#pragma unroll
      for (int w = 1; w < KW; ++w) acc[i] = acc[i] + partial[wave + w][i][lane];
  }
  // block i of C^T: lane holds columns 4 g .. 4 g + 3 of row l16
  if (l16 >= o.M) return;
  OUT *row = static_cast<OUT *>(o.C) + (size_t)l16 * o.N;
#pragma unroll
  for (int i = 0; i < UT; ++i) {
    const int n = n0 + i * 16 + g * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < o.N) {
        if constexpr (sizeof(OUT) == 2) row[n + e] = to_bf16(acc[i][e]);
        else row[n + e] = acc[i][e];
      }
  }
}

}  // namespace
}  // namespace occ
