// Types shared by the MX4 GEMM kernels (included by gemm_mx4.hip only).
#pragma once

#include "gemm_dl.h"
#include "mx4.h"

namespace occ {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// By value: a bit cast of a vector's element itself would read its first.
template <class T>
__device__ __forceinline__ T as_word(uint32_t w) {
  return __builtin_bit_cast(T, w);
}

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

// A tile of C leaves through LDS, so that its rows go to memory as whole runs: the 64-byte pieces of
// a row that the MFMA layout gives a wave cost 8192x8192x512 22 us of 67, and twice as much
// again where rows are not 64-byte aligned.
template <int BN, class OUT>
struct TileOut {
  static constexpr int PITCH = BN * (int)sizeof(OUT) + 16;  // bytes of a row in LDS
  // 16x16 block of C^T at (row, col) of the tile: lane l holds columns 4 (l / 16) .. + 3 of row l % 16
  static __device__ __forceinline__ void put(unsigned char *smem, int row, int col, int lane, f32x4 v) {
    unsigned char *p = smem + (row + (lane & 15)) * PITCH + (col + (lane >> 4) * 4) * (int)sizeof(OUT);
    if constexpr (sizeof(OUT) == 2) {
      *reinterpret_cast<uint64_t *>(p) = (uint64_t)pack_bf16(v[2], v[3]) << 32 | pack_bf16(v[0], v[1]);
    } else {
      *reinterpret_cast<f32x4 *>(p) = v;
    }
  }
  // ROWS rows from there to C's rows m0 .., columns n0 ..; NT threads
  template <int ROWS, int NT>
  static __device__ __forceinline__ void store(const unsigned char *smem, OUT *C, int M, int N, int m0, int n0) {
    typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2)));
    typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4)));
    typedef std::conditional_t<sizeof(OUT) == 2, u32x4_e2, u32x4_e4> u32x4_e;
    constexpr int E = 16 / (int)sizeof(OUT), CH = BN / E, RPP = NT / CH;  // elements a chunk, chunks a row, rows a pass
    static_assert(NT % CH == 0 && ROWS % RPP == 0, "whole rows per pass");
    const int row = threadIdx.x / CH, n = n0 + (int)(threadIdx.x % CH) * E;
#pragma unroll 4
    for (int r = row; r < ROWS; r += RPP) {
      if (m0 + r >= M) break;
      const u32x4 v = *reinterpret_cast<const u32x4 *>(smem + r * PITCH + (threadIdx.x % CH) * 16);
      OUT *c = C + (size_t)(m0 + r) * N + n;
      if (n + E <= N) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4_e *>(c));
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (n + e < N) {
            if constexpr (sizeof(OUT) == 2) c[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
            else c[e] = as_word<float>(v[e]);
          }
      }
    }
  }
};

}  // namespace
}  // namespace occ
