// Skinny (M <= 16) MX4 GEMM (included by gemm_mx4.hip only).
#pragma once

#include "gemm_mx4_common.h"

namespace occ {
namespace {

// ---------------------------------------------------------------------------
// M <= 16 (decode-like, bound by reading B once).  A unit is 16 columns of C (16 rows of B) over
// the whole K; KW waves of a workgroup take its 512-wide k-steps in turn, so that together
// they read KW * 256 contiguous bytes of every row, and 8 / KW units share a workgroup.
// Workgroups are persistent, two to a CU, and loop over units.
//
//  * A stays in registers: XS k-steps a wave (K <= 512 * KW * XS).  No load but B's is then
//    in the way of B's: loads return in order.
//  * A load takes 256 contiguous bytes of 4 rows; the k-step becomes operands through 4 KiB of
//    LDS that are the wave's own (chunks spread by row, no bank conflicts, no barrier),
//    which frees the registers for the next unit's loads before this one is
//    multiplied.  Read as operands lie, 64 bytes of each of 16 rows a load, with one
//    unit per workgroup, 16x28672x8192 took 32 us instead of 24.
//  * A lane's 16 bytes of an operand are one block of 32 columns; its word of the scale tile
//    serves all four MFMAs of the k-step.
//
// The KW partial sums are added in wave order through LDS (one of the waves each
// time, in turn): the result does not depend on timing.  Rows of A past M and of B
// past N lie beyond their descriptors and read as zero.
//
// NT: B's loads are non-temporal; chosen where B exceeds the L2s (see the launcher).
template <int KW, int XS, class OUT, bool NT>
__global__ __launch_bounds__(512, 4) void gemm_mx4_skinny_kernel(Mx4Operands o, int units) {
  constexpr int WPU = 8 / KW;
  __shared__ u32x4 staged[8][256];
  __shared__ f32x4 partial[2][8][64];
  extern __shared__ __align__(16) unsigned char pad_lds[];  // occupancy pad only
  (void)pad_lds;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave % KW, sub = wave / KW;
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t P = o.pitch;
  u32x4 *lds = staged[wave];
  constexpr int kPolicy = NT ? 2 : 0;

  u32x4 a[XS][4], b[XS][4];
  int as[XS], bs[XS];
  {
    const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.A), 0, (int)((uint32_t)o.M * P), 0x00020000);
    const auto ras = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.As), 0, (int)P, 0x00020000);
#pragma unroll
    for (int x = 0; x < XS; ++x) {
      const uint32_t k0 = (uint32_t)(kw + x * KW) * 256u;  // past K: beyond As, and no row of A either
#pragma unroll
      for (int s = 0; s < 4; ++s)
        a[x][s] = __builtin_amdgcn_raw_buffer_load_b128(
            ra, (int)(k0 < P ? (uint32_t)l16 * P + (uint32_t)g * 16u + k0 + s * 64u : 0x80000000u), 0, 0);
      as[x] = (int)__builtin_amdgcn_raw_buffer_load_b32(ras, (int)(lane * 4u + k0), 0, 0);
    }
  }
  auto load = [&](int unit) {
    const size_t n0 = (size_t)unit * 16;
    const int rows = min(16, o.N - unit * 16);
    const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.B) + n0 * P, 0, (int)((uint32_t)rows * P), 0x00020000);
    const auto rbs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.Bs) + (size_t)unit * P, 0, (int)P, 0x00020000);
#pragma unroll
    for (int x = 0; x < XS; ++x) {
      const uint32_t k0 = (uint32_t)(kw + x * KW) * 256u;
      if (k0 >= P) break;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        b[x][i] = __builtin_amdgcn_raw_buffer_load_b128(rb, (int)((uint32_t)g * P + (uint32_t)l16 * 16u + 4u * i * P),
                                                        (int)k0, kPolicy);
      bs[x] = (int)__builtin_amdgcn_raw_buffer_load_b32(rbs, lane * 4, (int)k0, kPolicy);
    }
  };

  const int step = (int)gridDim.x * WPU;
  int unit = (int)blockIdx.x * WPU + sub;
  const bool mine = (uint32_t)kw * 256u < P;  // this wave has a k-step
  if (unit < units) load(unit);
  int turn = 0, sums = 0;  // sums: which of the KW waves adds the parts
  for (int first = blockIdx.x * WPU; first < units; first += step, unit += step) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const bool live = unit < units;
    if (live && mine) {
      int scale[XS];
#pragma unroll
      for (int x = 0; x < XS; ++x) {
        scale[x] = bs[x];
        if (x > 0 && (uint32_t)(kw + x * KW) * 256u >= P) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[(4 * i + g) * 16 + (l16 ^ (4 * i + g))] = b[x][i];
        if (x == XS - 1 || (uint32_t)(kw + (x + 1) * KW) * 256u >= P) {  // all of b is in LDS or multiplied
          if (unit + step < units) load(unit + step);
          __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 w[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) w[s] = lds[l16 * 16 + ((4 * s + g) ^ l16)];
        acc = mfma_mx4<0>(w[0], a[x][0], acc, scale[x], as[x]);
        acc = mfma_mx4<1>(w[1], a[x][1], acc, scale[x], as[x]);
        acc = mfma_mx4<2>(w[2], a[x][2], acc, scale[x], as[x]);
        acc = mfma_mx4<3>(w[3], a[x][3], acc, scale[x], as[x]);
      }
    }
    bool store = live;
    if constexpr (KW > 1) {
      // partial[turn] was read two units ago, before a barrier that every writer has passed since
      if (live) partial[turn][wave][lane] = acc;
      __syncthreads();
      store = live && kw == sums;
      if (store) {
        acc = partial[turn][wave - kw][lane];
#pragma unroll
        for (int w = 1; w < KW; ++w) acc = acc + partial[turn][wave - kw + w][lane];
      }
      turn ^= 1;
      sums = sums + 1 == KW ? 0 : sums + 1;
    }
    // the unit of C^T: lane holds columns 4 g .. 4 g + 3 of row l16
    if (store && l16 < o.M) {
      const int n = unit * 16 + g * 4;
      OUT *c = static_cast<OUT *>(o.C) + (size_t)l16 * o.N + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < o.N) {
          if constexpr (sizeof(OUT) == 2) c[e] = to_bf16(acc[e]);
          else c[e] = acc[e];
        }
    }
  }
}

// The same for any K: A is read again, from the caches, for every unit of 32 columns, and a
// workgroup has one unit.  It keeps none of what makes the kernel above fast: 16 x 8192 x 28672 30 us and one row 24,
// where B's bytes are 21 (16 x 28672 x 8192 above: 24).
template <class OUT>
__global__ __launch_bounds__(512, 4) void gemm_mx4_skinny_long_kernel(Mx4Operands o) {
  constexpr int KW = 8, UT = 2, U = 2;
  __shared__ f32x4 partial[KW][UT][64];
  extern __shared__ __align__(16) unsigned char pad_lds[];  // occupancy pad only
  (void)pad_lds;
  const int lane = threadIdx.x & 63;
  const int kw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t P = o.pitch;
  const int n0 = (int)blockIdx.x * 16 * UT;
  const int nk = o.steps512;
  const int rows = min(16 * UT, o.N - n0);
  const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.B) + (size_t)n0 * P, 0, (int)((uint32_t)rows * P), 0x00020000);
  const auto rbs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.Bs) + (size_t)(n0 >> 4) * P, 0,
                                                     (int)((uint32_t)((rows + 15) >> 4) * P), 0x00020000);
  const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.A), 0, (int)((uint32_t)o.M * P), 0x00020000);
  const auto ras = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(o.As), 0, (int)P, 0x00020000);
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
          b[u][i][s] = __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(off + (uint32_t)(i * 16) * P + s * 64u + k0), 0, 0);
        bs[u][i] = (int)__builtin_amdgcn_raw_buffer_load_b32(rbs, (int)((uint32_t)i * P + lane * 4u + k0), 0, 0);
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
#pragma unroll
  for (int i = 0; i < UT; ++i) partial[kw][i][lane] = acc[i];
  __syncthreads();
  if (kw >= UT || l16 >= o.M) return;
  f32x4 v = partial[0][kw][lane];
#pragma unroll
  for (int w = 1; w < KW; ++w) v = v + partial[w][kw][lane];
  const int n = n0 + kw * 16 + g * 4;
  OUT *c = static_cast<OUT *>(o.C) + (size_t)l16 * o.N + n;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < o.N) {
      if constexpr (sizeof(OUT) == 2) c[e] = to_bf16(v[e]);
      else c[e] = v[e];
    }
}

}  // namespace
}  // namespace occ
