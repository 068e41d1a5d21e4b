// MX4 quantisation and its inverse (occ_mx4_quantize, occ_mx4_dequantize).
//
// q(x)_b = RNE_e2m1(x_b / 2^e), e = floor(log2(max |x_b|)) - 2 over blocks of 32.
// All that is computed is a maximum of exponents, but 10 to 20 instructions a word are near what the
// bytes take (2 or 4 in, 17/32 out per value and orientation).  8192 x 8192 bf16: rows 31 us
// (5.5 TB/s), both orientations 44 (4.7), back 26 (6.6); binary32: 58, 65 and 75 (5.2, 5.2, 4.0).
#include "block_util.h"
#include "mx4.h"

#include <algorithm>

namespace occ {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Magnitudes order as integers, a NaN above the infinities.  The largest of 8 values, as binary32 bits.
__device__ __forceinline__ uint32_t top_of(const Raw8<uint16_t> &r) {  // two values a word
  uint32_t t = r.w[0] & 0x7FFF7FFFu;
#pragma unroll
  for (int i = 1; i < 4; ++i) t = pk_max(t, r.w[i] & 0x7FFF7FFFu);
  return max(t << 16, t & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t top_of(const Raw8<float> &r) {
  uint32_t t = r.a[0] & 0x7FFFFFFFu;
#pragma unroll
  for (int i = 1; i < 8; ++i) t = max(t, (i < 4 ? r.a[i & 3] : r.b[i & 3]) & 0x7FFFFFFFu);
  return t;
}
// Over the lane and its 3 neighbours, whose 32 values are a block.
__device__ __forceinline__ uint32_t block_top(uint32_t t) {
  t = max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  return max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0x4E, 0xF, 0xF, true));  // lane ^ 2
}

// Codes of 8 values whose block has scale byte s: the hardware's conversion divides by the scale and
// rounds to nearest-even with saturation, as the format asks (checked on every scale and on ties).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t codes_of(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t s) {
  const float sc = mx4_scale_value(s);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w0), sc, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w1), sc, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w2), sc, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w3), sc, 3);
  return s == 255u ? 0u : c;
}
__device__ __forceinline__ uint32_t codes_of(const Raw8<uint16_t> &r, uint32_t s) {
  return codes_of(r.w[0], r.w[1], r.w[2], r.w[3], s);
}
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], uint32_t s) {
  const float sc = mx4_scale_value(s);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], sc, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], sc, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], sc, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], sc, 3);
  return s == 255u ? 0u : c;
}
__device__ __forceinline__ uint32_t codes_of(const Raw8<float> &r, uint32_t s) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r.at(e);
  return codes_of(v, s);
}

// ---------------------------------------------------------------------------
// Row blocks only.  A workgroup makes one scale tile at a time: 16 rows x 512 columns, a
// wave 4 rows, a lane 8 columns of each (4 lanes share a block's maximum through two
// lane swaps), the next tile's values on their way.  Loads are 1 or 2 KiB of a row per
// wave, codes 256 bytes, the tile's scales leave through LDS as 64 words.
template <class E>
__global__ __launch_bounds__(256) void mx4_quant_rows_kernel(const E *__restrict__ x, int rows, int cols, size_t ld,
                                                             uint8_t *__restrict__ codes, uint32_t *__restrict__ scales,
                                                             int tiles_c, int tiles) {
  __shared__ uint32_t words[2][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t pitch = (size_t)tiles_c * (kMx4Tile / 2);
  Raw8<E> v[4];
  auto load = [&](int tile) {
    const int t = tile / tiles_c, c = tile % tiles_c * kMx4Tile + lane * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = t * 16 + wave * 4 + i;
      const E *p = x + (size_t)row * ld + c;
      if (tile % tiles_c * kMx4Tile + kMx4Tile <= cols) v[i].load(p, row < rows);
      else v[i].load_part(p, row < rows ? cols - c : 0, cols);
    }
  };
  load(blockIdx.x);
  int turn = 0;
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1) {
    const int t = tile / tiles_c, c = tile % tiles_c * kMx4Tile + lane * 8;
    uint32_t code[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wave * 4 + i;
      const uint32_t sb = mx4_scale_of(block_top(top_of(v[i])));
      code[i] = codes_of(v[i], sb);
      if ((lane & 3) == 0) reinterpret_cast<uint8_t *>(words[turn])[mx4_scale_byte(r, lane >> 2)] = (uint8_t)sb;
    }
    if (tile + (int)gridDim.x < tiles) load(tile + gridDim.x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = t * 16 + wave * 4 + i;
      if (row < rows) *reinterpret_cast<uint32_t *>(codes + (size_t)row * pitch + (c >> 1)) = code[i];
    }
    __syncthreads();  // the words of two tiles ago have been read before this one's were written
    if (threadIdx.x < 64) scales[(size_t)tile * 64 + threadIdx.x] = words[turn][threadIdx.x];
  }
}

// ---------------------------------------------------------------------------
// Row and column blocks from one read, or column blocks alone.  A workgroup takes 128 x 128
// values: the rows are quantised as above on their way into LDS (16 lanes to a row), then
// each lane takes two neighbouring columns of 32 rows from there (one word per row
// of two bf16 values; two words for fp32).  The tiles of x are padded to whole scale
// tiles of the transpose (512 rows) and of x (512 columns), so that every code and scale of
// both outputs is written.
//
// Outputs leave in pieces of 64 bytes of a row and single scale bytes: the 16 tiles whose pieces
// share cache lines (512 x 512 values) go to one XCD one after the other, whose L2 joins them.
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
  // workgroups b, b + 8, b + 16, ... run on one XCD: 16 in a row of them are a 512 x 512 tile
  const int big = tiles_c * tiles_r, whole = big & ~7;
  int b = blockIdx.x, super, part;
  if (b < whole * 16) {
    super = (b >> 7) * 8 + (b & 7);
    part = (b >> 3) & 15;
  } else {
    super = b >> 4;
    part = b & 15;
  }
  const int r0 = (super / tiles_c * 4 + (part >> 2)) * 128, c0 = (super % tiles_c * 4 + (part & 3)) * 128;
  const size_t pitch = (size_t)tiles_c * 256, pitch_t = (size_t)tiles_r * 256;
  const int rl = threadIdx.x >> 4, cl = (threadIdx.x & 15) * 8, c = c0 + cl;
  const E *from = x + (size_t)(r0 + rl) * ld + c;  // the thread's rows are 16 apart
  const size_t step = 16 * ld;
  Raw8<E> v[8];
  // tiles whose columns all exist are spared a load's 24 selects: instructions bound this kernel (8192^2
  // bf16: 57 us with them and with every address multiplied out, now 44)
  if (c0 + 128 <= cols) {
#pragma unroll
    for (int p = 0; p < 8; ++p) v[p].load(from + p * step, r0 + p * 16 + rl < rows);
  } else {
#pragma unroll
    for (int p = 0; p < 8; ++p) v[p].load_part(from + p * step, r0 + p * 16 + rl < rows ? cols - c : 0, cols);
  }
  uint8_t *const codes_at = codes + (size_t)(r0 + rl) * pitch + (c >> 1);
  uint8_t *const scales_at = scales + (size_t)(r0 >> 4) * pitch + (size_t)(c >> 9) * 256 + mx4_scale_byte(rl, (c >> 5) & 15);
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int row = r0 + p * 16 + rl;
    u32x4 *q = reinterpret_cast<u32x4 *>(buf + (p * 16 + rl) * PITCH + cl * (int)sizeof(E));
    if constexpr (sizeof(E) == 2) {
      q[0] = v[p].w;
    } else {
      q[0] = v[p].a;
      q[1] = v[p].b;
    }
    if (codes != nullptr) {
      const uint32_t sb = mx4_scale_of(block_top(top_of(v[p])));
      if (row < rows) *reinterpret_cast<uint32_t *>(codes_at + p * 16 * pitch) = codes_of(v[p], sb);
      if ((lane & 3) == 0 && r0 + p * 16 < rows) scales_at[p * pitch] = (uint8_t)sb;
    }
  }
  __syncthreads();
  // wave w: rows 32 w .. 32 w + 31, lane: columns 2 lane, 2 lane + 1
  const int k = r0 + wave * 32;  // first column of this lane's blocks in the transpose
  uint32_t sb[2];
  u32x4 w[2];
  if constexpr (sizeof(E) == 2) {
    uint32_t v2[32], t = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      v2[i] = *reinterpret_cast<const uint32_t *>(buf + (wave * 32 + i) * PITCH + lane * 4);
      t = pk_max(t, v2[i] & 0x7FFF7FFFu);
    }
    sb[0] = mx4_scale_of(t << 16);
    sb[1] = mx4_scale_of(t & 0xFFFF0000u);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t lo[4], hi[4];  // a column's values of rows 8 d + 2 i, + 1
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_amdgcn_perm(v2[8 * d + 2 * i + 1], v2[8 * d + 2 * i], 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(v2[8 * d + 2 * i + 1], v2[8 * d + 2 * i], 0x07060302u);
      }
      w[0][d] = codes_of(lo[0], lo[1], lo[2], lo[3], sb[0]);
      w[1][d] = codes_of(hi[0], hi[1], hi[2], hi[3], sb[1]);
    }
  } else {
    float f[2][32];
    uint32_t t0 = 0, t1 = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const u32x2 q = *reinterpret_cast<const u32x2 *>(buf + (wave * 32 + i) * PITCH + lane * 8);
      f[0][i] = as_float(q[0]);
      f[1][i] = as_float(q[1]);
      t0 = max(t0, q[0] & 0x7FFFFFFFu);
      t1 = max(t1, q[1] & 0x7FFFFFFFu);
    }
    sb[0] = mx4_scale_of(t0);
    sb[1] = mx4_scale_of(t1);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = f[h][8 * d + i];
        w[h][d] = codes_of(e, sb[h]);
      }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = c0 + lane * 2 + h;  // row of the transpose
    if (row < cols) *reinterpret_cast<u32x4 *>(codes_t + (size_t)row * pitch_t + (k >> 1)) = w[h];
    if (row < (cols + 15) / 16 * 16)
      scales_t[(size_t)(row >> 4) * pitch_t + (size_t)(k >> 9) * 256 + mx4_scale_byte(row & 15, (k >> 5) & 15)] = (uint8_t)sb[h];
  }
}

// ---------------------------------------------------------------------------
// Values of codes, the way of mx4_quant_rows_kernel back: a scale tile at a time, a lane 8
// columns of 4 rows, the next tile's words on their way.  The conversion takes the scale byte
// as a binary32 exponent (0 is 2^-127, 255 makes NaN).
template <class E>
__global__ __launch_bounds__(256) void mx4_dequant_kernel(const uint8_t *__restrict__ codes,
                                                          const uint8_t *__restrict__ scales, int rows, int cols,
                                                          E *__restrict__ out, size_t ld, int tiles_c, int tiles) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t pitch = (size_t)tiles_c * (kMx4Tile / 2);
  uint32_t w[4], s[4];
  auto load = [&](int tile) {
    const int t = tile / tiles_c, c = tile % tiles_c * kMx4Tile + lane * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wave * 4 + i, row = min(t * 16 + r, rows - 1);
      w[i] = *reinterpret_cast<const uint32_t *>(codes + (size_t)row * pitch + (c >> 1));
      s[i] = scales[(size_t)tile * 256 + mx4_scale_byte(r, lane >> 2)];
    }
  };
  load(blockIdx.x);
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int t = tile / tiles_c, c = tile % tiles_c * kMx4Tile + lane * 8;
    uint32_t q[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = w[i], b[i] = s[i];
    if (tile + (int)gridDim.x < tiles) load(tile + gridDim.x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = t * 16 + wave * 4 + i;
      if (row >= rows || c >= cols) continue;
      const float sc = as_float(b[i] << 23);
      E *o = out + (size_t)row * ld + c;
      if constexpr (sizeof(E) == 2) {
        u32x4 p;
        p[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[i], sc, 0));
        p[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[i], sc, 1));
        p[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[i], sc, 2));
        p[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q[i], sc, 3));
        store_c_ragged(o, p, cols - c, false);
      } else {
        float v[8];
        const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], sc, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], sc, 1);
        const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], sc, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[i], sc, 3);
        v[0] = v0[0], v[1] = v0[1], v[2] = v1[0], v[3] = v1[1], v[4] = v2[0], v[5] = v2[1], v[6] = v3[0], v[7] = v3[1];
        if (cols - c >= 8) {
          store8<false>(o, true, v);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < cols - c) o[e] = v[e];
        }
      }
    }
  }
}

// Tiles of 16 x 512 that a launch's workgroups share: all resident at once.
unsigned tile_grid(int tiles, int num_cus) { return (unsigned)std::min(tiles, num_cus * 8); }

template <class E>
void launch_quant(const Mx4QuantCall &c, int num_cus, hipStream_t s) {
  const E *x = static_cast<const E *>(c.x);
  const int tiles_c = (c.cols + kMx4Tile - 1) / kMx4Tile, tiles_r = (c.rows + kMx4Tile - 1) / kMx4Tile;
  if (c.codes_t == nullptr) {
    const int tiles = (c.rows + 15) / 16 * tiles_c;
    hipLaunchKernelGGL(mx4_quant_rows_kernel<E>, dim3(tile_grid(tiles, num_cus)), dim3(256), 0, s, x, c.rows, c.cols,
                       c.ld, static_cast<uint8_t *>(c.codes), static_cast<uint32_t *>(c.scales), tiles_c, tiles);
    return;
  }
  const unsigned grid = (unsigned)(tiles_r * 4) * (unsigned)(tiles_c * 4);
  hipLaunchKernelGGL(mx4_quant_both_kernel<E>, dim3(grid), dim3(256), 0, s, x, c.rows, c.cols, c.ld,
                     static_cast<uint8_t *>(c.codes), static_cast<uint8_t *>(c.scales),
                     static_cast<uint8_t *>(c.codes_t), static_cast<uint8_t *>(c.scales_t), tiles_c, tiles_r);
}
}  // namespace

int mx4_quant_launch(const Mx4QuantCall &c, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  if (c.dtype == OCC_BF16) launch_quant<uint16_t>(c, di->num_cus, s);
  else launch_quant<float>(c, di->num_cus, s);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int mx4_dequant_launch(const Mx4DequantCall &c, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  const int tiles_c = (c.cols + kMx4Tile - 1) / kMx4Tile, tiles = (c.rows + 15) / 16 * tiles_c;
  const dim3 grid(tile_grid(tiles, di->num_cus));
  const uint8_t *codes = static_cast<const uint8_t *>(c.codes), *scales = static_cast<const uint8_t *>(c.scales);
  if (c.dtype == OCC_BF16)
    hipLaunchKernelGGL(mx4_dequant_kernel<uint16_t>, grid, dim3(256), 0, s, codes, scales, c.rows, c.cols,
                       static_cast<uint16_t *>(c.out), c.ld, tiles_c, tiles);
  else
    hipLaunchKernelGGL(mx4_dequant_kernel<float>, grid, dim3(256), 0, s, codes, scales, c.rows, c.cols,
                       static_cast<float *>(c.out), c.ld, tiles_c, tiles);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace occ
