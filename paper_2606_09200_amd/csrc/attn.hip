// Attention of new tokens over a paged cache (occ_attn_paged).
//
//   x_j = scale q . k_j for the keys j that the token sees;  m = max x_j,  p_j = exp(x_j - m),  l = sum p_j
//   o = sum p_j v_j / l,  lse = m + log l
//
// in one pass over the keys with the running m, l and o.  Two kernels, whose grid is the chip and whose workgroups
// take equal shares of the work (attn_plan.h); an item that several of them share is joined by the last to finish it, in
// the shares' order, so that results do not depend on who that is.
#include "attn_plan.h"
#include "block_util.h"
#include "divider.h"
#include "gemm_dl.h"
#include "once.h"

#include <algorithm>
#include <cmath>

namespace occ {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kDevice = 16;  // cache policy: device scope, as put_device
constexpr int kCus = 256;    // the workspace's size is asked for without a device
constexpr int kMaxDevices = 64;
constexpr int kFewRows = 64; // rows (tokens x heads of a group) of a request up to which the first kernel takes it
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 4 rows x 16 columns of 16-bit values in LDS, transposed: lane l of 16 gives the address of row l / 4, columns 4 (l %
// 4) .. + 3, and gets column l of the 4 rows.
__device__ __forceinline__ u32x2 read_transposed(uint32_t lds) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(size_t)lds));
}
__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(size_t)(__attribute__((address_space(3))) const unsigned char *)p;
}

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  return (int64_t)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

// The maximum and the sum over lanes l, l ^ 32 (and l ^ 16, l ^ 48), the same bits in all of them.
__device__ __forceinline__ float max_halves(float v) {
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return fmaxf(as_float(s[0]), as_float(s[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  return as_float(s[0]) + as_float(s[1]);
}
__device__ __forceinline__ float max_quarters(float v) {
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  return max_halves(fmaxf(as_float(s[0]), as_float(s[1])));
}
__device__ __forceinline__ float sum_quarters(float v) {
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  return sum_halves(as_float(s[0]) + as_float(s[1]));
}

// Whether one of two bf16 values is an infinity or a NaN, and the pair with such values zeroed.
__device__ __forceinline__ bool pair_nonfinite(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ uint32_t pair_finite(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
}

struct AttnCall {
  const uint16_t *q, *k, *v;
  const int32_t *table, *starts, *lens;
  uint16_t *out;
  float *lse;
  int n, rows, Hq, Hkv, D, group;
  int heads;           // of a tile, with its tokens cut.tokens of them
  int page, width, pages, keys;   // keys: width * page
  Divider by_page;
  size_t table_pitch;
  size_t q_row, q_head, out_row, out_head;           // elements
  size_t cache_page, cache_row, cache_head;
  float scale;         // of the exponent of 2
  AttnCut cut;
  int least, most;     // requests of `least` to `most` rows (tokens x heads of a group) are this launch's
  int min_share;
  uint32_t *joined;    // per share: finished parts of the item that begins in it
  float *part;
};

__device__ __forceinline__ AttnSeq seq_of(const AttnCall &c, int i) {
  AttnSeq s = attn_seq(c.starts[i], c.starts[i + 1], c.lens[i], c.rows, c.keys);
  const int64_t rows = (int64_t)s.fresh * c.group;
  if (rows < c.least || rows > c.most) s.fresh = 0;
  return s;
}

// Where a key's row lies in the caches (elements), and whether its page does.
struct KeyRow {
  int64_t at;
  bool bad;
};
__device__ __forceinline__ KeyRow key_row(const AttnCall &c, const int32_t *table, int key) {
  const int index = c.by_page(key);
  const int id = table[index];
  const bool bad = (uint32_t)id >= (uint32_t)c.pages;
  return KeyRow{(int64_t)(bad ? 0 : id) * (int64_t)c.cache_page + (int64_t)(key - index * c.page) * (int64_t)c.cache_row, bad};
}

struct WalkShared {
  int64_t wave[kWaves];
  int64_t at;
  int request;
  AttnSeq seq[kThreads];
};

// What a workgroup computes of an item: blocks [b0, b1) of 32 (64) keys from key `first` on, of which `last` is the end.
struct Piece {
  int request, part, tile;
  AttnSeq s;
  int first, last, b0, b1;
  AttnOwners owners;
  bool began;  // the item begins in this share
  bool alone;  // nobody else has a part of it
  bool first_began;  // it begins in the first share that has blocks of it
};

// Calls work(piece) for every item of this workgroup's share of the line.
template <class F>
__device__ __forceinline__ void walk(const AttnCall &c, WalkShared &sh, int me, int workgroups, F work) {
  const AttnCut &cut = c.cut;
  // units of all requests before each thread's own
  const int per = (c.n + kThreads - 1) / kThreads;
  const int r0 = min((int)threadIdx.x * per, c.n), r1 = min(r0 + per, c.n);
  int64_t own = 0;
  for (int i = r0; i < r1; ++i) {
    const AttnSeq s = seq_of(c, i);
    if (per == 1) sh.seq[threadIdx.x] = s;
    own += attn_units(cut, s);
  }
  int64_t upto = own;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t v = __shfl_up(upto, d);
    if ((int)(threadIdx.x & 63) >= d) upto += v;
  }
  if ((threadIdx.x & 63) == 63) sh.wave[threadIdx.x >> 6] = upto;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)(threadIdx.x >> 6)) upto += sh.wave[w];
    total += sh.wave[w];
  }
  total = uniform(total);
  const int64_t share = max((int64_t)c.min_share, (total + workgroups - 1) / workgroups);
  const int64_t lo = me * share, hi = min(lo + share, total);
  if (lo >= total) return;
  if (upto - own <= lo && lo < upto) {
    int64_t at = upto - own;
    int i = r0;
    for (; i < r1 - 1; ++i) {
      const int64_t u = attn_units(cut, per == 1 ? sh.seq[threadIdx.x] : seq_of(c, i));
      if (lo < at + u) break;
      at += u;
    }
    sh.request = i;
    sh.at = at;
  }
  __syncthreads();
  int i = uniform(sh.request), cached = 0;
  int64_t at_request = uniform(sh.at);
  bool filled = per == 1;
  for (; at_request < hi; ++i) {
    if (!filled || i >= cached + kThreads) {  // the next requests' lengths, one a thread
      __syncthreads();
      cached = i;
      if (cached + (int)threadIdx.x < c.n) sh.seq[threadIdx.x] = seq_of(c, cached + threadIdx.x);
      __syncthreads();
      filled = true;
    }
    AttnSeq s = sh.seq[i - cached];
    s.first = uniform(s.first), s.fresh = uniform(s.fresh), s.len = uniform(s.len);
    const int tiles = attn_tiles(cut, s);
    if (tiles == 0) continue;
    const int64_t units = attn_units_before(cut, s, tiles);
    const int64_t x = max(lo, at_request) - at_request;
    int part = x == 0 ? 0 : (int)(x / units);
    int m = x == 0 ? 0 : attn_tile_at(cut, s, x - part * units);
    AttnItem it;
    it.at = at_request + part * units + (m == 0 ? 0 : attn_units_before(cut, s, m));
    while (it.at < hi && part < cut.parts) {
      Piece p;
      p.request = i, p.part = part, p.tile = m, p.s = s;
      p.first = attn_first_key(cut, s, m), p.last = attn_last_key(cut, s, m);
      it.keys = p.last - p.first;
      p.b0 = attn_blocks_before(cut, it, lo), p.b1 = attn_blocks_before(cut, it, hi);
      p.owners = attn_owners(cut, it, share);
      p.began = it.at >= lo;
      p.first_began = it.at >= (int64_t)p.owners.from * share;
      p.alone = it.keys == 0 || p.owners.to - p.owners.from == 1;
      if (p.b0 < p.b1 || (it.keys == 0 && p.began)) work(p);
      it.at += cut.fixed + it.keys;
      if (++m == tiles) m = 0, ++part;
    }
    at_request += units * cut.parts;
  }
}

// A row of a tile: its token and head, and the keys [lo, hi) that it sees.
struct Row {
  int token, head, lo, hi;
  bool valid;
};
__device__ __forceinline__ Row row_of(const AttnCall &c, const Piece &p, int groups, int r) {
  const int t = r / c.heads, h = r - t * c.heads;
  const int token = p.tile * c.cut.tokens + t;
  const int kv = p.part / groups, in = (p.part - kv * groups) * c.heads + h;
  Row row;
  row.valid = t < c.cut.tokens && token < p.s.fresh && in < c.group;
  row.token = p.s.first + token;
  row.head = kv * c.group + in;
  const int pos = p.s.len - p.s.fresh + token;
  row.hi = !row.valid ? 0 : c.cut.causal ? min(pos + 1, p.s.len) : p.s.len;
  row.lo = c.cut.window ? pos - c.cut.window + 1 : 0;
  return row;
}
// Keys [all_lo, all_hi) that every row of a tile sees.
__device__ __forceinline__ void seen_by_all(const AttnCall &c, const Piece &p, int t0, int t1, int &all_lo, int &all_hi) {
  const int base = p.s.len - p.s.fresh + p.tile * c.cut.tokens;
  const int left = p.s.fresh - p.tile * c.cut.tokens;  // a tile's last tokens may not exist
  all_hi = c.cut.causal ? min(base + t0 + 1, p.s.len) : p.s.len;
  all_lo = c.cut.window ? base + min(t1, left) - c.cut.window : 0;
}

// ------------------------------------------------------------------ few rows
//
// Decoding: up to 16 rows (heads that share keys, times tokens) and many keys.  What bounds it is reading keys and
// values once.  Each of the workgroup's 4 waves takes every 4th block of 32 keys by itself, with no barrier: keys go
// from memory to the registers of S^T = K Q^T as they are (16x16x32 MFMAs: a lane holds 8 keys' scores of one row, which
// are what the second product wants of it), values pass through the wave's own LDS to be read transposed for O^T = V^T
// P^T.  P goes in as the sum of two bf16 values: matrix instructions are in plenty here, and o then has
// its own rounding alone.
template <int DP>
struct FewTile {
  static constexpr int ROWS = 16, KEYS = 32;
  static constexpr int KS = DP / 32, DT = DP / 16;
  static constexpr int PITCH = DP * 2;                 // bytes of a row of V in LDS
  static constexpr int O_PITCH = DP + 4;               // floats of a row of O there
  static constexpr int WAVE_BYTES = 64 * DP + 256;     // 32 rows of V, later 16 of O
  static constexpr int PART = ROWS * (DP + 2);         // floats of a partial result: O, then (m, l) of each row
  static constexpr int PER_CU = DP > 128 ? 1 : 2;
};

// Physical 16-byte chunk of chunk c in row r of the V tile.  Values are written 16 rows at a time at one chunk, and
// read 8 rows at a time in pieces of two chunks: both meet 16 different quarters of the 64 banks.
template <int DP>
__device__ __forceinline__ int few_swizzle(int r, int c) {
  if constexpr (DP >= 128) return c ^ ((r & 7) << 1) ^ ((r >> 3) & 1);
  else return c ^ (((r >> 1) & 3) << 1) ^ ((r >> 3) & 1);
}

template <int DP>
__global__ __launch_bounds__(kThreads, FewTile<DP>::PER_CU) void attn_few_kernel(AttnCall c) {
  using T = FewTile<DP>;
  constexpr int KS = T::KS, DT = T::DT;
  extern __shared__ __align__(256) unsigned char smem[];  // WAVE_BYTES a wave
  __shared__ WalkShared sh;
  __shared__ float ml[kWaves][2][16];
  __shared__ uint32_t last_one;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int l16 = lane & 15, g = lane >> 4;
  unsigned char *mine = smem + wave * T::WAVE_BYTES;
  const uint32_t mine_lds = lds_address(mine);
  const int groups = c.cut.parts / c.Hkv;

  walk(c, sh, (int)xcd_remap(blockIdx.x, gridDim.x), (int)gridDim.x, [&](const Piece &p) {
    const int kv = p.part / groups;
    const Row row = row_of(c, p, groups, l16);
    int all_lo, all_hi;
    seen_by_all(c, p, 0, c.cut.tokens, all_lo, all_hi);
    const int32_t *table = c.table + (size_t)p.request * c.table_pitch;
    const uint16_t *kc = c.k + (size_t)kv * c.cache_head + 8 * g, *vc = c.v + (size_t)kv * c.cache_head + 8 * g;

    u32x4 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = u32x4{0u, 0u, 0u, 0u};
      if (row.valid && 32 * s + 8 * g < c.D)
        q[s] = *reinterpret_cast<const u32x4 *>(c.q + (size_t)row.token * c.q_row + (size_t)row.head * c.q_head + 32 * s + 8 * g);
    }
    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    for (int b = p.b0 + wave; b < p.b1; b += kWaves) {
      const int kb = p.first + b * T::KEYS;
      u32x4 k[2][KS], v[2][KS];
      uint64_t bad[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const KeyRow r = key_row(c, table, min(kb + 16 * t + l16, p.last - 1));
        bad[t] = __ballot(r.bad);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          k[t][s] = v[t][s] = u32x4{0u, 0u, 0u, 0u};
          if (32 * s + 8 * g < c.D) {
            k[t][s] = *reinterpret_cast<const u32x4 *>(kc + r.at + 32 * s);
            v[t][s] = *reinterpret_cast<const u32x4 *>(vc + r.at + 32 * s);
          }
        }
      }
      f32x4 x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) x[t] = mfma16(k[t][s], q[s], x[t]);
      }
      // a lane's scores are of keys 16 t + 4 g + i
      const bool masked = kb < all_lo || kb + T::KEYS > all_hi || ((bad[0] | bad[1]) & 0xFFFFu) != 0;
      if (masked) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 16 * t + 4 * g + i;
            const bool seen = kb + at >= row.lo && kb + at < row.hi && !((bad[t] >> (4 * g + i)) & 1u);
            x[t][i] = seen ? x[t][i] : -INFINITY;
          }
      }
      float top = x[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
      top = fmaxf(m, max_quarters(top) * c.scale);
      const float by = top == -INFINITY ? 0.f : top;
      const float less = exp2_(m - by);
      m = top;
      l = l * less;
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = exp2_(__builtin_fmaf(x[i >> 2][i & 3], c.scale, -by));
        l = l + e[i];
      }
      u32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = pack_bf16(e[2 * i], e[2 * i + 1]);
        lo[i] = pack_bf16(e[2 * i] - bf16_lo(hi[i]), e[2 * i + 1] - bf16_hi(hi[i]));
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] = acc[t] * less;
      // values: 16 rows at one chunk at a time
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int r = 16 * t + l16;
          *reinterpret_cast<u32x4 *>(mine + r * T::PITCH + few_swizzle<DP>(r, 4 * s + g) * 16) = v[t][s];
        }
      asm volatile("" ::: "memory");  // the wave's LDS accesses are served in order
      const int vr = 4 * g + (l16 >> 2);
      const uint32_t v0 = mine_lds + vr * T::PITCH + few_swizzle<DP>(vr, (l16 & 3) >> 1) * 16 + 8 * (l16 & 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const uint32_t at = (v0 ^ ((t & 7) * 32)) + (t >> 3) * 256;
        const u32x2 a = read_transposed(at), b2 = read_transposed(at + 16 * T::PITCH);
        u32x4 vt = {a[0], a[1], b2[0], b2[1]};
        // a value that a row does not see must not reach it, whatever it is, and one that it sees must not meet the
        // lower half of a weight, which may be 0: infinities and NaN go in one by one
        const bool odd = pair_nonfinite(vt[0]) || pair_nonfinite(vt[1]) || pair_nonfinite(vt[2]) || pair_nonfinite(vt[3]);
        if (__ballot(odd) != 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) vt[i] = pair_finite(vt[i]);
#pragma unroll 1
          for (int r = 0; r < T::KEYS; ++r) {
            const uint64_t w = *reinterpret_cast<const uint64_t *>(
                mine + r * T::PITCH + few_swizzle<DP>(r, 2 * t + (g >> 1)) * 16 + 8 * (g & 1));
            const bool seen = kb + r >= row.lo && kb + r < row.hi && !((bad[r >> 4] >> (r & 15)) & 1u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t h = (uint32_t)(w >> (16 * i)) & 0xFFFFu;
              if (seen && (h & 0x7F80u) == 0x7F80u) acc[t][i] = acc[t][i] + as_float(h << 16);
            }
          }
        }
        acc[t] = mfma16(vt, hi, acc[t]);
        acc[t] = mfma16(vt, lo, acc[t]);
      }
      asm volatile("" ::: "memory");
    }

    // the waves' results, joined
    l = sum_quarters(l);
    if (g == 0) ml[wave][0][l16] = m, ml[wave][1][l16] = l;
    float *o = reinterpret_cast<float *>(mine);
#pragma unroll
    for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4 *>(o + l16 * T::O_PITCH + 16 * t + 4 * g) = acc[t];
    __syncthreads();
    constexpr int CH = DP / 8;  // pieces of 8 values in a row
    const int slots = (int)gridDim.x * 2;
    const auto rs = rsrc_of(c.part, (uint32_t)(slots * T::PART * 4));
    const int me = (int)xcd_remap(blockIdx.x, gridDim.x);
    auto finish = [&](int r, int ch, const float (&v)[8], float top, float sum) {
      const Row w = row_of(c, p, groups, r);
      if (!w.valid) return;
      const float by = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
      if (8 * ch < c.D) {
        u32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = pack_bf16(v[2 * i] * by, v[2 * i + 1] * by);
        *reinterpret_cast<u32x4 *>(c.out + (size_t)w.token * c.out_row + (size_t)w.head * c.out_head + 8 * ch) = h;
      }
      if (ch == 0 && c.lse != nullptr)
        c.lse[(size_t)w.token * c.Hq + w.head] = sum > 0.f || sum != sum ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    };
    for (int e = threadIdx.x; e < 16 * CH; e += kThreads) {
      const int r = e / CH, ch = e % CH;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][0][r]);
      const float by = top == -INFINITY ? 0.f : top;
      float sum = 0.f, v[8] = {};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_(ml[w][0][r] - by);
        sum = __builtin_fmaf(ml[w][1][r], f, sum);
        const float *ow = reinterpret_cast<const float *>(smem + w * T::WAVE_BYTES) + r * T::O_PITCH + 8 * ch;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf(ow[i], f, v[i]);
      }
      if (p.alone) {
        finish(r, ch, v, top, sum);
      } else {
        const uint32_t slot = (uint32_t)(2 * me + (p.began ? 1 : 0)) * (T::PART * 4);
        const uint32_t at = slot + (uint32_t)(r * DP + 8 * ch) * 4u;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}), rs, (int)at, 0, kDevice);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}), rs, (int)at + 16, 0, kDevice);
        if (ch == 0)
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{top, sum}), rs,
                                                (int)(slot + (uint32_t)(16 * DP + 2 * r) * 4u), 0, kDevice);
      }
    }
    if (!p.alone) {
      stores_done();
      const int parts = p.owners.to - p.owners.from;
      if (threadIdx.x == 0) {
        const bool last = add_device(c.joined + p.owners.from) + 1 == (uint32_t)parts;
        if (last) put_device(c.joined + p.owners.from, 0u);  // for the next call
        last_one = last;
      }
      __syncthreads();
      if (last_one != 0u) {
        for (int e = threadIdx.x; e < 16 * CH; e += kThreads) {
          const int r = e / CH, ch = e % CH;
          float top = -INFINITY, sum = 0.f, v[8] = {};
          for (int w0 = 0; w0 < parts; w0 += 4) {
            f32x4 a[4], b[4];
            f32x2 t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int w = p.owners.from + min(w0 + j, parts - 1);
              // the item's first part may be of a share that it begins in
              const uint32_t slot = (uint32_t)(2 * w + (w == p.owners.from && p.first_began ? 1 : 0)) * (T::PART * 4);
              const uint32_t at = slot + (uint32_t)(r * DP + 8 * ch) * 4u;
              a[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at, 0, kDevice));
              b[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at + 16, 0, kDevice));
              t[j] = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(slot + (uint32_t)(16 * DP + 2 * r) * 4u), 0, kDevice));
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (w0 + j >= parts) break;
              const float now = fmaxf(top, t[j][0]), by = now == -INFINITY ? 0.f : now;
              const float f0 = exp2_(top - by), f1 = exp2_(t[j][0] - by);
              top = now;
              sum = __builtin_fmaf(t[j][1], f1, sum * f0);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                v[i] = __builtin_fmaf(a[j][i], f1, v[i] * f0);
                v[4 + i] = __builtin_fmaf(b[j][i], f1, v[4 + i] * f0);
              }
            }
          }
          finish(r, ch, v, top, sum);
        }
      }
    }
    __syncthreads();
  });
}

// ------------------------------------------------------------------ many rows
//
// Chunks of a prompt: 128 rows (tokens times heads that share keys) of a workgroup's 4 waves, 32 each, against
// tiles of 64 keys that direct-to-LDS loads bring in while the tile before is multiplied.  S^T = K Q^T in 32x32x16
// MFMAs leaves a lane 16 keys' scores of one row (the other half of the wave has the other 16), which,
// rounded to bf16, are the second product's operand as they lie: O^T = V^T P^T over the keys in that order, values
// read transposed.  m and l are one register a lane, and so is what o has to be scaled by.  The weights' rounding (8
// bits) is of the same size as the output's own; l sums them unrounded.
template <int DP>
struct ManyTile {
  static constexpr int ROWS = 128, KEYS = 64;
  static constexpr int KS = DP / 16, DT = DP / 32;
  static constexpr int CH = DP / 8;                    // 16-byte chunks of a row
  static constexpr int PITCH = DP * 2;
  static constexpr int OPERAND = KEYS * PITCH;         // bytes of a tile of K, and of V
  static constexpr int STAGE = 2 * OPERAND;
  static constexpr int PASS_ROWS = kThreads / CH, PASSES = KEYS / PASS_ROWS;
  static constexpr int PART = ROWS * (DP + 2);
  static constexpr int PER_CU = DP > 128 ? 1 : 2;
};

// Physical chunk of chunk c in row r: a read of K sends 16 rows at one chunk, one of V, by 32 lanes, 4 rows at 4
// chunks in a row.
template <int DP>
__device__ __forceinline__ int many_swizzle_k(int r, int c) {
  if constexpr (DP >= 128) return c ^ (r & 15);
  else return swz<8>(r, c);
}
template <int DP>
__device__ __forceinline__ int many_swizzle_v(int r, int c) {
  return swz_kn<ManyTile<DP>::CH>(r, c);
}

// 16 bytes a lane from its own address to LDS at `lds` + 16 lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void global_dma16(const void *from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from)
               : "memory", "m0");
}
#pragma clang diagnostic pop

template <int DP>
__global__ __launch_bounds__(kThreads, ManyTile<DP>::PER_CU) void attn_many_kernel(AttnCall c) {
  using T = ManyTile<DP>;
  constexpr int KS = T::KS, DT = T::DT;
  extern __shared__ __align__(256) unsigned char stages[];
  __shared__ WalkShared sh;
  __shared__ uint32_t bad_rows[3][2];
  __shared__ uint32_t last_one;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
  const uint32_t lds0 = lds_address(stages);
  const int groups = c.cut.parts / c.Hkv;
  const int slots = (int)gridDim.x * 2;
  const auto rs = rsrc_of(c.part, (uint32_t)slots * (uint32_t)(T::PART * 4));
  const int me = (int)xcd_remap(blockIdx.x, gridDim.x);

  // chunks that the heads do not have stay zero
  if (c.D < DP)
    for (int i = threadIdx.x; i < 2 * T::STAGE / 16; i += kThreads) reinterpret_cast<u32x4 *>(stages)[i] = u32x4{0u, 0u, 0u, 0u};
  if (threadIdx.x < 6) (&bad_rows[0][0])[threadIdx.x] = 0u;
  __syncthreads();

  walk(c, sh, me, (int)gridDim.x, [&](const Piece &p) {
    const int kv = p.part / groups;
    const Row row = row_of(c, p, groups, wave * 32 + l32);
    int all_lo, all_hi;
    seen_by_all(c, p, wave * 32 / c.heads, (wave * 32 + 31) / c.heads + 1, all_lo, all_hi);
    const int32_t *table = c.table + (size_t)p.request * c.table_pitch;
    const uint16_t *kc = c.k + (size_t)kv * c.cache_head, *vc = c.v + (size_t)kv * c.cache_head;
    const int r_in = threadIdx.x / T::CH, chunk = threadIdx.x % T::CH;

    auto issue = [&](int b) {
      const int stage = b & 1, flags = b % 3;
      const uint32_t to = lds0 + (uint32_t)stage * T::STAGE + (uint32_t)wave * 1024u;
#pragma unroll
      for (int i = 0; i < T::PASSES; ++i) {
        const int r = i * T::PASS_ROWS + r_in;
        const KeyRow kr = key_row(c, table, min(p.first + b * T::KEYS + r, p.last - 1));
        if (kr.bad && chunk == 0) atomicOr(&bad_rows[flags][r >> 5], 1u << (r & 31));
        const int ck = many_swizzle_k<DP>(r, chunk), cv = many_swizzle_v<DP>(r, chunk);
        if (8 * ck < c.D) global_dma16(kc + kr.at + 8 * ck, to + (uint32_t)i * 4096u);
        if (8 * cv < c.D) global_dma16(vc + kr.at + 8 * cv, to + T::OPERAND + (uint32_t)i * 4096u);
      }
    };

    u32x4 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = u32x4{0u, 0u, 0u, 0u};
      if (row.valid && 16 * s + 8 * half < c.D)
        q[s] = *reinterpret_cast<const u32x4 *>(c.q + (size_t)row.token * c.q_row + (size_t)row.head * c.q_head + 16 * s + 8 * half);
    }
    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;

    if (p.b0 < p.b1) issue(p.b0);
    for (int b = p.b0; b < p.b1; ++b) {
      wait_vmcnt<0>();
      __syncthreads();  // tile b has landed, and nobody reads the one before any more
      if (threadIdx.x < 2) bad_rows[(b + 2) % 3][threadIdx.x] = 0u;
      if (b + 1 < p.b1) issue(b + 1);
      const int kb = p.first + b * T::KEYS;
      const uint32_t kt = lds0 + (uint32_t)(b & 1) * T::STAGE, vt0 = kt + T::OPERAND;
      const uint32_t bad0 = bad_rows[b % 3][0], bad1 = bad_rows[b % 3][1];
      f32x16 x[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[t][i] = 0.f;
        const uint32_t at = kt + (uint32_t)((32 * t + l32) * T::PITCH + many_swizzle_k<DP>(l32, half) * 16);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const uint32_t a = (at ^ ((s & 7) * 32)) + (s >> 3) * 256;
          const u32x4 k = *(__attribute__((address_space(3))) const u32x4 *)(size_t)a;
          x[t] = mfma32(k, q[s], x[t]);
        }
      }
      // a lane's scores are of keys 32 t + 8 (i / 4) + 4 half + i % 4
      const bool masked = kb < all_lo || kb + T::KEYS > all_hi || uniform((int)(bad0 | bad1)) != 0;
      if (masked) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int at = 8 * (i >> 2) + 4 * half + (i & 3);
            const bool seen = kb + 32 * t + at >= row.lo && kb + 32 * t + at < row.hi && !(((t ? bad1 : bad0) >> at) & 1u);
            x[t][i] = seen ? x[t][i] : -INFINITY;
          }
      }
      float top = x[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, x[i >> 4][i & 15]);
      top = fmaxf(m, max_halves(top) * c.scale);
      const float by = top == -INFINITY ? 0.f : top;
      const float less = exp2_(m - by);
      m = top;
      l = l * less;
      u32x4 w[4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float e0 = exp2_(__builtin_fmaf(x[t][2 * i], c.scale, -by)), e1 = exp2_(__builtin_fmaf(x[t][2 * i + 1], c.scale, -by));
          l = l + (e0 + e1);
          w[2 * t + (i >> 2)][i & 3] = pack_bf16(e0, e1);
        }
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] = acc[t] * less;
      const int vr = 4 * half + (l16 >> 2);
      const uint32_t v0 = vt0 + vr * T::PITCH + many_swizzle_v<DP>(vr, 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) * 16 + 8 * (l16 & 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        u32x4 vt[4];
        const uint32_t at = (v0 ^ ((t & 3) * 64)) + (t >> 2) * 256;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const u32x2 a = read_transposed(at + 16 * s * T::PITCH), b2 = read_transposed(at + (16 * s + 8) * T::PITCH);
          vt[s] = u32x4{a[0], a[1], b2[0], b2[1]};
        }
        if (masked) {
          // a value that a row does not see must not reach it, whatever it is: infinities and NaN go in one by one
          bool odd = false;
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) odd = odd || pair_nonfinite(vt[s][i]);
          if (__ballot(odd) != 0) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
              for (int i = 0; i < 4; ++i) vt[s][i] = pair_finite(vt[s][i]);
#pragma unroll 1
            for (int r = 0; r < T::KEYS; ++r) {
              const bool seen = kb + r >= row.lo && kb + r < row.hi && !(((r & 32 ? bad1 : bad0) >> (r & 31)) & 1u);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                // values 32 t + 8 i + 4 half .. + 3 of key r
                const uint32_t a = vt0 + r * T::PITCH + many_swizzle_v<DP>(r, 4 * t + i) * 16 + 8 * half;
                const u32x2 h = *(__attribute__((address_space(3))) const u32x2 *)(size_t)a;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const uint32_t f = ((j & 2 ? h[1] : h[0]) >> (16 * (j & 1))) & 0xFFFFu;
                  if (seen && (f & 0x7F80u) == 0x7F80u) acc[t][4 * i + j] = acc[t][4 * i + j] + as_float(f << 16);
                }
              }
            }
          }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[t] = mfma32(vt[s], w[s], acc[t]);
      }
    }
    l = sum_halves(l);

    const int r = wave * 32 + l32;
    if (!p.alone) {
      const uint32_t slot = (uint32_t)(2 * me + (p.began ? 1 : 0)) * (uint32_t)(T::PART * 4);
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 v = {acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs,
                                                 (int)(slot + (uint32_t)(r * DP + 32 * t + 8 * i + 4 * half) * 4u), 0, kDevice);
        }
      if (half == 0)
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{m, l}), rs,
                                              (int)(slot + (uint32_t)(T::ROWS * DP + 2 * r) * 4u), 0, kDevice);
      stores_done();
      const int parts = p.owners.to - p.owners.from;
      if (threadIdx.x == 0) {
        const bool last = add_device(c.joined + p.owners.from) + 1 == (uint32_t)parts;
        if (last) put_device(c.joined + p.owners.from, 0u);  // for the next call
        last_one = last;
      }
      __syncthreads();
      if (last_one != 0u) {
        m = -INFINITY, l = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
#pragma unroll 1
        for (int s = 0; s < parts; ++s) {
          const int from = p.owners.from + s;
          const uint32_t slot = (uint32_t)(2 * from + (s == 0 && p.first_began ? 1 : 0)) * (uint32_t)(T::PART * 4);
          const f32x2 t2 = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(slot + (uint32_t)(T::ROWS * DP + 2 * r) * 4u), 0, kDevice));
          const float now = fmaxf(m, t2[0]), by = now == -INFINITY ? 0.f : now;
          const float f0 = exp2_(m - by), f1 = exp2_(t2[0] - by);
          m = now;
          l = __builtin_fmaf(t2[1], f1, l * f0);
#pragma unroll
          for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                  rs, (int)(slot + (uint32_t)(r * DP + 32 * t + 8 * i + 4 * half) * 4u), 0, kDevice));
#pragma unroll
              for (int j = 0; j < 4; ++j) acc[t][4 * i + j] = __builtin_fmaf(v[j], f1, acc[t][4 * i + j] * f0);
            }
        }
      }
    }
    if ((p.alone || last_one != 0u) && row.valid) {
      const bool some = l > 0.f || l != l;
      const float by = some ? 1.f / l : 0.f;
      uint16_t *to = c.out + (size_t)row.token * c.out_row + (size_t)row.head * c.out_head;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = 32 * t + 8 * i + 4 * half;
          if (d < c.D)
            *reinterpret_cast<u32x2 *>(to + d) = u32x2{pack_bf16(acc[t][4 * i] * by, acc[t][4 * i + 1] * by),
                                                       pack_bf16(acc[t][4 * i + 2] * by, acc[t][4 * i + 3] * by)};
        }
      if (half == 0 && c.lse != nullptr)
        c.lse[(size_t)row.token * c.Hq + row.head] = some ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
    __syncthreads();
    if (threadIdx.x < 6) (&bad_rows[0][0])[threadIdx.x] = 0u;
    __syncthreads();
  });
}

// ------------------------------------------------------------------ launches

// Workgroups of a launch: what the chip holds at once.
int workgroups_of(bool many, int DP, int cus) {
  return cus * (many ? (DP > 128 ? ManyTile<256>::PER_CU : ManyTile<128>::PER_CU) : (DP > 128 ? FewTile<256>::PER_CU : FewTile<128>::PER_CU));
}
int padded_head(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <int DP, bool MANY>
int launch(const AttnCall &c, int grid, hipStream_t s) {
  void (*fn)(AttnCall);
  if constexpr (MANY) fn = attn_many_kernel<DP>;
  else fn = attn_few_kernel<DP>;
  constexpr int lds = MANY ? 2 * ManyTile<DP>::STAGE : kWaves * FewTile<DP>::WAVE_BYTES;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return OCC_ENODEV;
  static Once limit_set[kMaxDevices];
  if (!limit_set[dev].run([&] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
      }))
    return OCC_EHIP;
  hipLaunchKernelGGL(fn, dim3(grid), dim3(kThreads), lds, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}
template <bool MANY>
int launch(const AttnCall &c, int DP, int grid, hipStream_t s) {
  return DP == 64 ? launch<64, MANY>(c, grid, s) : DP == 128 ? launch<128, MANY>(c, grid, s) : launch<256, MANY>(c, grid, s);
}

constexpr int kJoined = 2 * kCus;  // shares, at most

}  // namespace

size_t attn_workspace(int D) {
  const int DP = padded_head(D);
  const size_t few = (size_t)workgroups_of(false, DP, kCus) * 2 * FewTile<128>::ROWS * (DP + 2) * 4;
  const size_t many = (size_t)workgroups_of(true, DP, kCus) * 2 * ManyTile<128>::ROWS * (DP + 2) * 4;
  return (size_t)kJoined * 4 + std::max(few, many);
}

int attn_launch(const occ_attn_args &a, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (a.requests == 0 || a.rows == 0) return OCC_OK;
  AttnCall c{};
  c.q = static_cast<const uint16_t *>(a.q), c.k = static_cast<const uint16_t *>(a.k_cache), c.v = static_cast<const uint16_t *>(a.v_cache);
  c.table = a.table, c.starts = a.starts, c.lens = a.lens;
  c.out = static_cast<uint16_t *>(a.out), c.lse = a.lse;
  c.n = a.requests, c.rows = a.rows, c.Hq = a.Hq, c.Hkv = a.Hkv, c.D = a.D, c.group = a.Hq / a.Hkv;
  c.page = a.page, c.width = a.width, c.pages = a.pages;
  c.keys = (int)std::min<int64_t>((int64_t)a.width * a.page, OCC_ATTN_MAX_KEYS);
  c.by_page = Divider(a.page);
  c.table_pitch = a.ld_table;
  c.q_row = a.q_row, c.q_head = a.q_head, c.out_row = a.out_row, c.out_head = a.out_head;
  c.cache_page = a.cache_page, c.cache_row = a.cache_row, c.cache_head = a.cache_head;
  c.scale = a.scale * kLog2e;
  c.joined = static_cast<uint32_t *>(a.workspace);
  c.part = reinterpret_cast<float *>(static_cast<unsigned char *>(a.workspace) + (size_t)kJoined * 4);
  const int DP = padded_head(a.D), cus = std::min(di->num_cus, kCus);
  auto go = [&](bool many, int least, int most) {
    AttnCall k = c;
    const int rows = many ? ManyTile<128>::ROWS : FewTile<128>::ROWS;
    k.heads = std::min(c.group, rows);
    k.cut.tokens = rows / k.heads;
    k.cut.parts = a.Hkv * ((c.group + k.heads - 1) / k.heads);
    k.cut.fixed = many ? 64 : 32, k.cut.block = many ? ManyTile<128>::KEYS : FewTile<128>::KEYS;
    k.cut.window = a.window, k.cut.causal = a.causal != 0;
    k.least = least, k.most = most;
    k.min_share = 256;
    const int grid = workgroups_of(many, DP, cus);
    return many ? launch<true>(k, DP, grid, s) : launch<false>(k, DP, grid, s);
  };
  const int most_rows = (int)std::min<int64_t>((int64_t)std::min(a.max_fresh, a.rows) * c.group, INT32_MAX);
  if (most_rows <= kFewRows) return go(false, 0, INT32_MAX);
  // all requests of the largest size, as far as the host can know
  if (a.requests == 1 || (int64_t)a.requests * a.max_fresh == a.rows) return go(true, 0, INT32_MAX);
  const int few = go(false, 0, kFewRows);
  return few == OCC_OK ? go(true, kFewRows + 1, INT32_MAX) : few;
}

}  // namespace occ
