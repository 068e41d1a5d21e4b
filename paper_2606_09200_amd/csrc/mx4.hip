// MX4 quantisation and its inverse (occ_mx4_quantize, occ_mx4_dequantize).
//
// q(x)_b = RNE_e2m1(x_b / 2^e), e = floor(log2(max |x_b|)) - 2 over blocks of 32.
// All that is computed is a maximum of exponents; both kernels are bound by the
// bytes they move (2 or 4 in, 17/32 out per value and orientation).
#include "block_util.h"
#include "mx4.h"

namespace occ {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t mag(float f) { return __builtin_bit_cast(uint32_t, f) & 0x7FFFFFFFu; }

// Largest magnitude of 8 values and of the 3 neighbouring lanes' (a block of 32), as
// bits: magnitudes order as integers, and a NaN is above the infinities.
__device__ __forceinline__ uint32_t block_top(const float (&v)[8]) {
  uint32_t t = mag(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) t = max(t, mag(v[i]));
  t = max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  t = max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0x4E, 0xF, 0xF, true));  // lane ^ 2
  return t;
}

// ---------------------------------------------------------------------------
// Row blocks only.  A workgroup makes one scale tile: 16 rows x 512 columns, a
// wave 4 rows, a lane 8 columns of each (4 lanes share a block's maximum through
// two lane swaps).  Loads are 1 or 2 KiB of a row per wave, codes 256 bytes, the
// tile's scales leave through LDS as 64 words.
template <class E>
__global__ __launch_bounds__(256) void mx4_quant_rows_kernel(const E *__restrict__ x, int rows, int cols, size_t ld,
                                                             uint8_t *__restrict__ codes, uint32_t *__restrict__ scales,
                                                             int tiles_c) {
  __shared__ uint32_t tile[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x / tiles_c, s = blockIdx.x % tiles_c;
  const int c = s * kMx4Tile + lane * 8;
  const size_t pitch = (size_t)tiles_c * (kMx4Tile / 2);
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = t * 16 + wave * 4 + i;
    load8(x + (size_t)min(row, rows - 1) * ld + min(c, cols), row < rows ? cols - c : 0, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = wave * 4 + i, row = t * 16 + r;
    const uint32_t sb = mx4_scale_of(block_top(v[i]));
    if (row < rows) *reinterpret_cast<uint32_t *>(codes + (size_t)row * pitch + (c >> 1)) = mx4_codes8(v[i], sb);
    if ((lane & 3) == 0) reinterpret_cast<uint8_t *>(tile)[mx4_scale_byte(r, lane >> 2)] = (uint8_t)sb;
  }
  __syncthreads();
  if (threadIdx.x < 64) scales[(size_t)blockIdx.x * 64 + threadIdx.x] = tile[threadIdx.x];
}

// ---------------------------------------------------------------------------
// Row and column blocks from one read, or column blocks alone.  A workgroup takes
// 128 x 128 values: the rows are quantised as above on their way into LDS (16 lanes
// to a row), then each lane reads two neighbouring columns of 32 rows from there (one
// word per row of two bf16 values; two words for fp32).  Grid: the tiles of x padded to
// whole scale tiles of the transpose (512 rows) and of x (512 columns), so that
// every code and scale of both outputs is written.
template <class E>
struct QuantBoth {
  static constexpr int PITCH = 128 * (int)sizeof(E) + 16;  // bytes of a row in LDS
};

template <class E>
__global__ __launch_bounds__(256) void mx4_quant_both_kernel(const E *__restrict__ x, int rows, int cols, size_t ld,
                                                             uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                             uint8_t *__restrict__ codes_t,
                                                             uint8_t *__restrict__ scales_t, int tiles_c, int tiles_r) {
  constexpr int PITCH = QuantBoth<E>::PITCH;
  __shared__ __align__(16) unsigned char buf[128 * PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nc = tiles_c * 4;  // 128-column tiles
  const int tr = blockIdx.x / nc, tc = blockIdx.x % nc;
  const int r0 = tr * 128, c0 = tc * 128;
  const size_t pitch = (size_t)tiles_c * 256, pitch_t = (size_t)tiles_r * 256;
  const int cl = (threadIdx.x & 15) * 8, c = c0 + cl;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int rl = p * 16 + (threadIdx.x >> 4), row = r0 + rl;
    float v[8];
    load8(x + (size_t)min(row, rows - 1) * ld + min(c, cols), row < rows ? cols - c : 0, v);
    unsigned char *q = buf + rl * PITCH + cl * (int)sizeof(E);
    if constexpr (sizeof(E) == 2) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i)  // bf16 values as binary32: the upper halves are their bits
        w[i] = (__builtin_bit_cast(uint32_t, v[2 * i]) >> 16) | (__builtin_bit_cast(uint32_t, v[2 * i + 1]) & 0xFFFF0000u);
      *reinterpret_cast<u32x4 *>(q) = w;
    } else {
      *reinterpret_cast<f32x4 *>(q) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4 *>(q + 16) = f32x4{v[4], v[5], v[6], v[7]};
    }
    if (codes != nullptr) {
      const uint32_t sb = mx4_scale_of(block_top(v));
      if (row < rows) *reinterpret_cast<uint32_t *>(codes + (size_t)row * pitch + (c >> 1)) = mx4_codes8(v, sb);
      if ((lane & 3) == 0 && row < (rows + 15) / 16 * 16)
        scales[(size_t)(row >> 4) * pitch + (size_t)(c >> 9) * 256 + mx4_scale_byte(row & 15, (c >> 5) & 15)] = (uint8_t)sb;
    }
  }
  __syncthreads();
  // wave w: rows 32 w .. 32 w + 31, lane: columns 2 lane, 2 lane + 1
  float v[2][32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const unsigned char *q = buf + (wave * 32 + i) * PITCH + lane * 2 * (int)sizeof(E);
    if constexpr (sizeof(E) == 2) {
      const uint32_t w = *reinterpret_cast<const uint32_t *>(q);
      v[0][i] = bf16_lo(w);
      v[1][i] = bf16_hi(w);
    } else {
      const u32x2 w = *reinterpret_cast<const u32x2 *>(q);
      v[0][i] = as_float(w[0]);
      v[1][i] = as_float(w[1]);
    }
  }
  const int k = r0 + wave * 32;  // first column of this lane's blocks in the transpose
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = c0 + lane * 2 + h;  // row of the transpose
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, mag(v[h][i]));
    const uint32_t sb = mx4_scale_of(top);
    u32x4 w;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = v[h][8 * d + i];
      w[d] = mx4_codes8(e, sb);
    }
    if (row < cols) *reinterpret_cast<u32x4 *>(codes_t + (size_t)row * pitch_t + (k >> 1)) = w;
    if (row < (cols + 15) / 16 * 16)
      scales_t[(size_t)(row >> 4) * pitch_t + (size_t)(k >> 9) * 256 + mx4_scale_byte(row & 15, (k >> 5) & 15)] = (uint8_t)sb;
  }
}

// ---------------------------------------------------------------------------
// Values of codes: a lane takes 8 columns (one word of codes, 16 or 32 bytes out).
template <class E>
__global__ __launch_bounds__(256) void mx4_dequant_kernel(const uint8_t *__restrict__ codes,
                                                          const uint8_t *__restrict__ scales, int rows, int cols,
                                                          E *__restrict__ out, size_t ld, int tiles_c) {
  const size_t pitch = (size_t)tiles_c * 256;
  const int per_row = (cols + 7) / 8;
  const size_t n = (size_t)rows * per_row;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const int row = (int)(i / per_row), c = (int)(i % per_row) * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + (size_t)row * pitch + (c >> 1));
    const uint32_t s = scales[(size_t)(row >> 4) * pitch + (size_t)(c >> 9) * 256 + mx4_scale_byte(row & 15, (c >> 5) & 15)];
    const float sc = mx4_scale_value(s);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t q = (w >> (4 * e)) & 15u, m = q & 7u;
      // E2M1 as binary32: codes 2..7 are exponent and fraction bits, 1 is 0.5
      const uint32_t b = m >= 2u ? ((m >> 1) + 126u) << 23 | (m & 1u) << 22 : m == 1u ? 0x3F000000u : 0u;
      v[e] = __builtin_bit_cast(float, b | (q >> 3) << 31) * sc;
    }
    store8(out + (size_t)row * ld + c, cols - c, v);
  }
}

template <class E>
void launch_quant(const Mx4QuantCall &c, hipStream_t s) {
  const E *x = static_cast<const E *>(c.x);
  const int tiles_c = (c.cols + kMx4Tile - 1) / kMx4Tile, tiles_r = (c.rows + kMx4Tile - 1) / kMx4Tile;
  if (c.codes_t == nullptr) {
    const unsigned grid = (unsigned)((c.rows + 15) / 16) * (unsigned)tiles_c;
    hipLaunchKernelGGL(mx4_quant_rows_kernel<E>, dim3(grid), dim3(256), 0, s, x, c.rows, c.cols, c.ld,
                       static_cast<uint8_t *>(c.codes), static_cast<uint32_t *>(c.scales), tiles_c);
    return;
  }
  const unsigned grid = (unsigned)(tiles_r * 4) * (unsigned)(tiles_c * 4);
  hipLaunchKernelGGL(mx4_quant_both_kernel<E>, dim3(grid), dim3(256), 0, s, x, c.rows, c.cols, c.ld,
                     static_cast<uint8_t *>(c.codes), static_cast<uint8_t *>(c.scales),
                     static_cast<uint8_t *>(c.codes_t), static_cast<uint8_t *>(c.scales_t), tiles_c, tiles_r);
}

}  // namespace

int mx4_quant_launch(const Mx4QuantCall &c, hipStream_t s) {
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  if (c.dtype == OCC_BF16) launch_quant<uint16_t>(c, s);
  else launch_quant<float>(c, s);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int mx4_dequant_launch(const Mx4DequantCall &c, hipStream_t s) {
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  const int tiles_c = (c.cols + kMx4Tile - 1) / kMx4Tile;
  const size_t n = (size_t)c.rows * ((c.cols + 7) / 8), wgs = (n + 255) / 256;
  const unsigned grid = (unsigned)(wgs < 16384 ? wgs : 16384);
  const uint8_t *codes = static_cast<const uint8_t *>(c.codes), *scales = static_cast<const uint8_t *>(c.scales);
  if (c.dtype == OCC_BF16)
    hipLaunchKernelGGL(mx4_dequant_kernel<uint16_t>, dim3(grid), dim3(256), 0, s, codes, scales, c.rows, c.cols,
                       static_cast<uint16_t *>(c.out), c.ld, tiles_c);
  else
    hipLaunchKernelGGL(mx4_dequant_kernel<float>, dim3(grid), dim3(256), 0, s, codes, scales, c.rows, c.cols,
                       static_cast<float *>(c.out), c.ld, tiles_c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace occ
