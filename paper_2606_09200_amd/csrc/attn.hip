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

// Two values as bf16 in one instruction.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
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

// Bits 0x80008000 are set where one of two bf16 values is an infinity or a NaN; the pair with such values zeroed.
__device__ __forceinline__ uint32_t pair_exponents(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
__device__ __forceinline__ uint32_t pair_finite(uint32_t w) {
  return ((w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u);
}

// Whether some row's maximum is one that exact_maximum is for.
__device__ __forceinline__ bool large_maximum(float by) { return __ballot(fabsf(by) >= 0x1p24f && fabsf(by) < INFINITY) != 0; }
// Scores of a row whose maximum is `by` (in powers of 2) as exponents, exp2 (scale x - by): the product goes into the difference
// unrounded, the maximum is a rounded one.  From 2^24 on that is off by 1 and more, by 2^7 at 2^31, and no weight would be left, or an
// infinite one: there x becomes what, times scale, is the difference of rounded products, 0 at the maximum, and `by` 0.
template <int TILES, class Acc>
__device__ __forceinline__ void exact_maximum(Acc (&x)[TILES], float scale, float &by) {
  const bool large = fabsf(by) >= 0x1p24f;
  const float back = 1.f / scale;  // of numbers above 2^24 / 2^128 where it is used
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Acc) / 4); ++i) x[t][i] = large ? (x[t][i] * scale - by) * back : x[t][i];
  by = large ? 0.f : by;
}

struct AttnCall {
  const uint16_t *q, *k, *v;
  const int32_t *table, *starts, *lens;
  uint16_t *out;
  float *lse;
  int n, rows, Hq, Hkv, D, group;
  int heads;           // of a tile, with its tokens cut.tokens of them
  int groups;          // of heads that share keys, tiles' heads at a time
  Divider by_heads, by_groups;
  int page, width, pages, keys;   // keys: width * page
  Divider by_page;
  size_t table_pitch;
  size_t q_row, q_head, out_row, out_head;           // elements
  size_t cache_head;
  uint32_t page_bytes, row_bytes;                    // of the caches
  float scale;         // of the exponent of 2
  AttnCut cut;
  int least, most;     // requests of `least` to `most` rows (tokens x heads of a group) are this launch's
  int min_share, least_even, spare;
  uint32_t *joined;    // per share: finished parts of the item that begins in it
  float *part;
};

__device__ __forceinline__ AttnSeq seq_of(const AttnCall &c, int i) {
  AttnSeq s = attn_seq(c.starts[i], c.starts[i + 1], c.lens[i], c.rows, c.keys);
  const int64_t rows = (int64_t)s.fresh * c.group;
  if (rows < c.least || rows > c.most) s.fresh = 0;
  return s;
}

// A launch argument in registers of its own: one spilled with its neighbours costs a read of each.
template <class V>
__device__ __forceinline__ V own_register(V v) {
  asm volatile("" : "+s"(v));
  return v;
}

// Where keys' rows lie in the caches.
struct KeyRows {
  Divider by_page;
  int page, pages;
  uint32_t page_bytes, row_bytes;
  __device__ __forceinline__ explicit KeyRows(const AttnCall &c)
      : by_page(c.by_page), page(own_register(c.page)), pages(own_register(c.pages)), page_bytes(own_register(c.page_bytes)),
        row_bytes(own_register(c.row_bytes)) {
    by_page.mul = own_register(by_page.mul), by_page.shift = own_register(by_page.shift);
  }
  __device__ __forceinline__ int page_of(int key) const { return by_page(key); }
  // A page that is none counts as the first: what is read there is not used.
  __device__ __forceinline__ bool bad(int id) const { return (uint32_t)id >= (uint32_t)pages; }
  // Bytes from a cache's beginning to row `off` of page `id`.
  __device__ __forceinline__ uint64_t at(int id, int off) const {
    return (uint64_t)(bad(id) ? 0u : (uint32_t)id) * page_bytes + (uint64_t)(uint32_t)off * row_bytes;
  }
};
template <class V>
__device__ __forceinline__ const V *plus(const void *p, uint64_t bytes) {
  return reinterpret_cast<const V *>(static_cast<const char *>(p) + bytes);
}

template <int THREADS>
struct WalkShared {
  int64_t sums[2][THREADS / 64];
  int64_t at;
  int request;
  uint32_t last_one;
  AttnSeq seq[THREADS];
};

// What a workgroup computes of an item: blocks [b0, b1) of the keys from `first` on, of which `last` is the end.
struct Piece {
  int request, kv, group, tile;
  AttnSeq s;
  AttnItem it;
  int first, last, b0, b1;
  bool began;  // the item begins in this share
  bool alone;  // nobody else has a part of it
  int even;    // workgroups that have an even part of it, from `base` on; 0: the item is on the line
  int base;
};

// Sums of two numbers of each thread over the threads before it, and over all.
template <int THREADS>
__device__ __forceinline__ void block_sums(WalkShared<THREADS> &sh, int64_t (&v)[2], int64_t (&total)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t upto[2] = {sum_upto(v[0]), sum_upto(v[1])};
  if (lane == 63) sh.sums[0][wave] = upto[0], sh.sums[1][wave] = upto[1];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    total[n] = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) upto[n] += sh.sums[n][w];
      total[n] += sh.sums[n][w];
    }
    total[n] = uniform(total[n]);
    v[n] = upto[n] - v[n];
  }
}

// a / b for 0 <= a < 1024 and b >= 1: half a unit from a whole number, which is more than the reciprocal is off by.
__device__ __forceinline__ int quotient(int a, int b) { return uniform((int)(((float)a + 0.5f) * __builtin_amdgcn_rcpf((float)b))); }

// What workgroup `me` of `shares` has to do, piece by piece: the same in all its threads, which call together.
template <int THREADS, bool FLAT>
struct Walk {
  const AttnCall &c;
  WalkShared<THREADS> &sh;
  AttnCut cut;
  AttnShare share;
  Piece p;
  // on the line: the next item, of request p.request, and the end of the share
  int64_t lo, hi, at, at_request, units, tile_units;
  int per, cached, tiles, part;
  bool left;  // something is left to do

  __device__ __forceinline__ void request(int i) {
    p.request = i;
    if (per > 1 && (cached < 0 || i >= cached + THREADS)) {  // the next requests' lengths, one a thread
      __syncthreads();
      cached = i;
      if (cached + (int)threadIdx.x < c.n) sh.seq[threadIdx.x] = seq_of(c, cached + threadIdx.x);
      __syncthreads();
    }
    p.s = sh.seq[per > 1 ? i - cached : i];
    p.s.first = uniform(p.s.first), p.s.fresh = uniform(p.s.fresh), p.s.len = uniform(p.s.len);
    tiles = attn_tiles(cut, p.s);
  }
  __device__ __forceinline__ void item(int which, int tile) {
    p.kv = c.by_groups(which), p.group = which - p.kv * c.groups, p.tile = tile;
    p.first = attn_first_key(cut, p.s, tile), p.last = attn_last_key(cut, p.s, tile);
    p.it.keys = p.last - p.first;
  }

  __device__ __forceinline__ Walk(const AttnCall &c_, WalkShared<THREADS> &sh_, int me, int shares) : c(c_), sh(sh_), cut(c_.cut) {
    cut.flat = FLAT;
    left = false, cached = -1, part = 0;
    p.even = 0, p.base = 0, p.tile = 0;
    // units and items of all requests before each thread's own
    per = (c.n + THREADS - 1) / THREADS;
    const int r0 = min((int)threadIdx.x * per, c.n), r1 = min(r0 + per, c.n);
    int64_t own[2] = {0, 0}, before[2], total[2];
#pragma unroll 1
    for (int i = r0; i < r1; ++i) {
      const AttnSeq s = seq_of(c, i);
      if (per == 1) sh.seq[threadIdx.x] = s;
      own[0] += attn_units(cut, s);
      own[1] += (int64_t)cut.parts * attn_tiles(cut, s);
    }
    before[0] = own[0], before[1] = own[1];
    block_sums(sh, before, total);
    if (total[1] == 0) return;  // a launch that has none of a step's requests
    // where even parts are better, the sums are of parts
    int even = attn_even_units(total[0] - total[1] * cut.fixed, total[1], shares, c.least_even, c.spare);
    auto size = [&](const AttnSeq &s) {
      return even == 0 ? attn_units(cut, s) : (int64_t)cut.parts * attn_tiles(cut, s) * attn_even_parts(attn_most_keys(cut, s), even);
    };
    if (even != 0) {
      int64_t parts = 0, first[2] = {0, 0}, all[2];
#pragma unroll 1
      for (int i = r0; i < r1; ++i) parts += size(per == 1 ? sh.seq[threadIdx.x] : seq_of(c, i));
      first[0] = parts;
      __syncthreads();  // the sums before have been read
      block_sums(sh, first, all);
      if (all[0] <= shares) own[0] = parts, before[0] = first[0], total[0] = all[0];
      else even = 0;  // tiles of a request may be shorter than its longest
    }
    if (even != 0) {
      lo = me, hi = me + 1;
    } else {
      share = attn_share(total[0], shares, c.min_share);
      share.units = uniform(share.units);
      lo = me * share.units, hi = min(lo + share.units, total[0]);
    }
    if (lo >= total[0]) return;
    if (before[0] <= lo && lo < before[0] + own[0]) {
      int64_t from = before[0];
      int i = r0;
#pragma unroll 1
      for (; i < r1 - 1; ++i) {
        const int64_t u = size(seq_of(c, i));
        if (lo < from + u) break;
        from += u;
      }
      sh.request = i;
      sh.at = from;
    }
    __syncthreads();
    left = true;
    at = at_request = uniform(sh.at);
    request(uniform(sh.request));
    if (even != 0) {
      const int k = attn_even_parts(attn_most_keys(cut, p.s), even), in = (int)(lo - at);
      const int which = quotient(in, k), j = in - which * k;
      part = quotient(which, tiles);
      item(part, which - part * tiles);
      const int blocks = (p.it.keys + cut.block - 1) / cut.block;
      p.b0 = attn_even_blocks(blocks, k, j), p.b1 = attn_even_blocks(blocks, k, j + 1);
      p.even = k, p.base = me - j;
      p.began = true, p.alone = min(blocks, k) <= 1;
      left = p.b0 < p.b1 || (blocks == 0 && j == 0);
      return;
    }
    units = attn_units_before(cut, p.s, tiles);
    tile_units = attn_units_before(cut, p.s, 1);  // of every tile, where that is the same
    if (lo > at) {  // from within the request
      while (at + units <= lo) at += units, ++part;
      if (FLAT) {
        p.tile = AttnShare{tile_units, 1.0 / (double)tile_units}(lo - at);
        at += p.tile * tile_units;
      } else {
        p.tile = attn_tile_at(cut, p.s, lo - at);
        if (p.tile > 0) at += attn_units_before(cut, p.s, p.tile);
      }
    }
  }

  // The next piece in `p`; false where there is none.
  __device__ __forceinline__ bool next() {
    if (!left) return false;
    if (p.even != 0) {
      left = false;
      return true;
    }
#pragma unroll 1
    while (at < hi) {
      if (part == cut.parts) {  // of the next request that has items
        at_request += units * cut.parts;
        do request(p.request + 1);
        while (tiles == 0);
        units = attn_units_before(cut, p.s, tiles);
        tile_units = attn_units_before(cut, p.s, 1);
        part = 0, p.tile = 0;
      }
      const int tile = p.tile;
      item(part, tile);
      p.it.at = at;
      p.b0 = attn_blocks_before(cut, p.it, lo), p.b1 = attn_blocks_before(cut, p.it, hi);
      p.began = at >= lo;
      p.alone = p.b0 == 0 && p.b1 * cut.block >= p.it.keys;
      at += FLAT ? tile_units : cut.fixed + p.it.keys;
      following = tile + 1;
      if (following == tiles) following = 0, ++part;
      if (p.b0 < p.b1 || (p.it.keys == 0 && p.began)) return true;
      p.tile = following;
    }
    return false;
  }
  __device__ __forceinline__ void done() { p.tile = following; }
  int following = 0;
};

// The workgroups that have a part of an item: how many, and where the first keeps the item's counter.
struct Joining {
  int counter, parts;
  bool even;
  bool in_first;  // the line: the item begins in the first share that has blocks of it
};
__device__ __forceinline__ Joining joining(const AttnCall &c, const Piece &p, const AttnShare &share) {
  Joining j;
  j.even = p.even != 0, j.in_first = true;
  if (p.even != 0) {
    j.counter = p.base, j.parts = min((p.it.keys + c.cut.block - 1) / c.cut.block, p.even);
  } else {
    const AttnOwners o = attn_owners(c.cut, p.it, share);
    j.counter = uniform(o.from), j.parts = uniform(o.to) - j.counter;
    j.in_first = p.it.at >= (int64_t)j.counter * share.units;
  }
  return j;
}

// Whether this workgroup, its part of the item stored, is the last of those that have one (the same in all threads).
template <int THREADS>
__device__ __forceinline__ bool last_of(const AttnCall &c, WalkShared<THREADS> &sh, const Joining &j) {
  stores_done();
  if (threadIdx.x == 0) {
    const bool last = add_device(c.joined + j.counter) + 1 == (uint32_t)j.parts;
    if (last) put_device(c.joined + j.counter, 0u);  // for the next call
    sh.last_one = last;
  }
  __syncthreads();
  return sh.last_one != 0u;
}

// Whether all others have theirs already, as it is where the item's end is a share's first piece and its beginning another's
// last: then this one's need not be stored (8 us for 256 rows of 128, of 17 to 20 us that a join took with it).
template <int THREADS>
__device__ __forceinline__ bool others_done(const AttnCall &c, WalkShared<THREADS> &sh, const Joining &j) {
  if (threadIdx.x == 0) {
    const bool last = get_device(c.joined + j.counter) + 1 == (uint32_t)j.parts;
    if (last) put_device(c.joined + j.counter, 0u);
    sh.last_one = last;
  }
  __syncthreads();
  const bool last = sh.last_one != 0u;
  __syncthreads();
  return last;
}

// Places of partial results: two a workgroup, for an item that began before its share and for one that begins in it.
__device__ __forceinline__ uint32_t place_of(int share, bool began, int floats) { return (uint32_t)(2 * share + (began ? 1 : 0)) * (uint32_t)(floats * 4); }

__device__ __forceinline__ uint32_t place_of(const Joining &j, int part, int floats) {
  return place_of(j.counter + part, j.even || (part == 0 && j.in_first), floats);
}

// A row of a tile: its token and head, and the keys [lo, hi) that it sees.
struct Row {
  int token, head, lo, hi;
  bool valid;
};
__device__ __forceinline__ Row row_of(const AttnCall &c, const Piece &p, int r) {
  const int t = c.by_heads(r), h = r - t * c.heads;
  const int in = p.group * c.heads + h;
  const AttnRow of = attn_row(c.cut, p.s, p.tile, t);
  Row row;
  row.valid = t < c.cut.tokens && of.valid && in < c.group;
  row.token = p.s.first + of.token;
  row.head = p.kv * c.group + in;
  row.lo = of.lo, row.hi = row.valid ? of.hi : 0;
  return row;
}
// ------------------------------------------------------------------ few rows
//
// Decoding: up to 16 rows (heads that share keys, times tokens) and many keys.  What bounds it is reading keys and
// values once.  Each of the workgroup's 8 waves takes every 8th block of 32 keys by itself, with no barrier: keys go
// from memory to the registers of S^T = K Q^T as they are (16x16x32 MFMAs: a lane holds 8 keys' scores of one row, which
// are what the second product wants of it), values pass through the wave's own LDS to be read transposed for O^T = V^T
// P^T.  P goes in as the sum of two bf16 values: matrix instructions are in plenty here, and o then has
// its own rounding alone (off by 0.0016 of its size; 0.0023 with one).
//   Heads of 256 take a register more than there are: it is spilled before the loop and read again behind it.
//   One workgroup a CU, so that a share is long: 64 requests of 1 to 8191 keys, 64 heads over 8 of 128, 214 us (5.0 TB/s; a
// copy has 4.95, mostly reads 5.8), 40 heads of their own 250 (5.3 TB/s); 130000 keys of one request 117 (4.55 TB/s: workgroups finish 70 to 96 us
// after they begin, as their pages lie).  Four requests of 500 keys 13: 3.6 the plan, 3 pages and keys, 4 the parts' way
// through memory, 2.3 a launch.
template <int DP>
struct FewTile {
  static constexpr int WAVES = 8, THREADS = 64 * WAVES;
  static constexpr int ROWS = 16, TILES = DP > 128 ? 1 : 2, KEYS = 16 * TILES;
  static constexpr int KS = DP / 32, DT = DP / 16;
  static constexpr int PITCH = DP * 2;                 // bytes of a row of V in LDS
  static constexpr int O_PITCH = DP + 4;               // floats of a row of O there
  static constexpr int WAVE_BYTES = 64 * DP + 256;     // KEYS rows of V, later 16 of O
  static constexpr int PART = ROWS * (DP + 2);         // floats of a partial result: O, then (m, l) of each row
  static constexpr int PER_CU = 1;
};

// Physical 16-byte chunk of chunk c in row r of the V tile.  Values are written 16 rows at a time at one chunk, and
// read 8 rows at a time in pieces of two chunks: both meet 16 different quarters of the 64 banks.
template <int DP>
__device__ __forceinline__ int few_swizzle(int r, int c) {
  if constexpr (DP >= 128) return c ^ ((r & 7) << 1) ^ ((r >> 3) & 1);
  else return c ^ (((r >> 1) & 3) << 1) ^ ((r >> 3) & 1);
}

template <int DP>
__global__ __launch_bounds__(FewTile<DP>::THREADS, FewTile<DP>::PER_CU) void attn_few_kernel(AttnCall c) {
  using T = FewTile<DP>;
  constexpr int KS = T::KS, DT = T::DT, TILES = T::TILES;
  extern __shared__ __align__(256) unsigned char smem[];  // WAVE_BYTES a wave
  __shared__ WalkShared<T::THREADS> sh;
  __shared__ float ml[T::WAVES][2][16];
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6));
  const int l16 = lane & 15, g = lane >> 4;
  unsigned char *mine = smem + wave * T::WAVE_BYTES;
  const uint32_t mine_lds = lds_address(mine);
  const KeyRows rows(c);
  const int me = (int)blockIdx.x;

  Walk<T::THREADS, true> walk(c, sh, me, (int)gridDim.x);
#pragma unroll 1
  for (; walk.next(); walk.done()) {
    const Piece &p = walk.p;
    const Row row = row_of(c, p, l16);
    const auto [all_lo, all_hi] = attn_all_see(c.cut, p.s, p.tile, 0, c.cut.tokens);  // keys that every row sees
    const int32_t *table = c.table + (size_t)p.request * c.table_pitch;
    const uint16_t *kc = c.k + (size_t)p.kv * c.cache_head + 8 * g, *vc = c.v + (size_t)p.kv * c.cache_head + 8 * g;

    // A block's keys are asked for when the ones before have been multiplied, its values when those have gone to LDS: one
    // set of registers each, and something in flight at all times.  The page numbers of the block after
    // are asked for before either, so that waiting for them does not wait for these.
    u32x4 k[TILES][KS], v[TILES][KS];
    int ids[TILES], keys[TILES], pages[TILES];
    uint64_t at[TILES];
    uint32_t bad = 0, next_bad = 0;  // a bit for each key of the block whose page is none
    auto ask = [&](int b) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        keys[t] = min(p.first + b * T::KEYS + 16 * t + l16, p.last - 1);
        pages[t] = rows.page_of(keys[t]);
        ids[t] = table[pages[t]];
      }
    };
    auto load = [&](u32x4 (&to)[TILES][KS], const uint16_t *from) {
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          to[t][s] = u32x4{0u, 0u, 0u, 0u};
          if (32 * s + 8 * g < c.D) to[t][s] = *plus<u32x4>(from + 32 * s, at[t]);
        }
    };
    auto load_keys = [&](int b) {
      next_bad = 0;
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        at[t] = rows.at(ids[t], keys[t] - pages[t] * rows.page);
        next_bad |= ((uint32_t)__ballot(rows.bad(ids[t])) & 0xFFFFu) << (16 * t);
      }
      if (b + T::WAVES < p.b1) ask(b + T::WAVES);
      load(k, kc);
    };
    if (p.b0 + wave < p.b1) ask(p.b0 + wave);
    u32x4 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = u32x4{0u, 0u, 0u, 0u};
      if (row.valid && 32 * s + 8 * g < c.D)
        q[s] = *reinterpret_cast<const u32x4 *>(c.q + (size_t)row.token * c.q_row + (size_t)row.head * c.q_head + 32 * s + 8 * g);
    }
    if (p.b0 + wave < p.b1) {
      load_keys(p.b0 + wave);
      load(v, vc);
    }
    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

#pragma unroll 1
    for (int b = p.b0 + wave; b < p.b1; b += T::WAVES) {
      const int kb = p.first + b * T::KEYS;
      const bool more = b + T::WAVES < p.b1;
      bad = next_bad;
      f32x4 x[TILES];
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) x[t] = mfma16(k[t][s], q[s], x[t]);
      }
      if (more) load_keys(b + T::WAVES);
      // a lane's scores are of keys 16 t + 4 g + i
      if (kb < all_lo || kb + T::KEYS > all_hi || bad != 0) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = 16 * t + 4 * g + i;
            const bool seen = kb + key >= row.lo && kb + key < row.hi && !((bad >> key) & 1u);
            x[t][i] = seen ? x[t][i] : -INFINITY;
          }
      }
      float top = x[0][0];
#pragma unroll
      for (int i = 1; i < 4 * TILES; ++i) top = fmaxf(top, x[i >> 2][i & 3]);
      top = fmaxf(m, max_quarters(top) * c.scale);
      float by = top == -INFINITY ? 0.f : top;
      const float less = exp2_(m - by);
      m = top;
      if (large_maximum(by)) exact_maximum(x, c.scale, by);
      l = l * less;
      float e[8] = {};
#pragma unroll
      for (int i = 0; i < 4 * TILES; ++i) {
        e[i] = exp2_(__builtin_fmaf(x[i >> 2][i & 3], c.scale, -by));
        l = l + e[i];
      }
      u32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = pack2(e[2 * i], e[2 * i + 1]);
        lo[i] = pack2(e[2 * i] - bf16_lo(hi[i]), e[2 * i + 1] - bf16_hi(hi[i]));
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] = acc[t] * less;
      // values: 16 rows at one chunk at a time
      auto put_values = [&]() {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            const int r = 16 * t + l16;
            *reinterpret_cast<u32x4 *>(mine + r * T::PITCH + few_swizzle<DP>(r, 4 * s + g) * 16) = v[t][s];
          }
        asm volatile("" ::: "memory");  // the wave's LDS accesses are served in order
      };
      put_values();
      // a value that a row does not see must not reach it, whatever it is, and one that it sees must not meet the
      // lower half of a weight, which may be 0: infinities and NaN go in one by one
      uint32_t odd = 0;
#pragma unroll
      for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= pair_exponents(v[t][s][i]);
      if (__ballot((odd & 0x80008000u) != 0) != 0) {
#pragma unroll 1
        for (int r = 0; r < T::KEYS; ++r) {
          const bool seen = kb + r >= row.lo && kb + r < row.hi && !((bad >> r) & 1u);
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            const uint64_t four = *reinterpret_cast<const uint64_t *>(
                mine + r * T::PITCH + few_swizzle<DP>(r, 2 * t + (g >> 1)) * 16 + 8 * (g & 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t h = (uint32_t)(four >> (16 * i)) & 0xFFFFu;
              if (seen && (h & 0x7F80u) == 0x7F80u) acc[t][i] = acc[t][i] + as_float(h << 16);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[t][s][i] = pair_finite(v[t][s][i]);
        put_values();
      }
      if (more) load(v, vc);
      const int vr = 4 * g + (l16 >> 2);
      const uint32_t v0 = mine_lds + vr * T::PITCH + few_swizzle<DP>(vr, (l16 & 3) >> 1) * 16 + 8 * (l16 & 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const uint32_t from = (v0 ^ ((t & 7) * 32)) + (t >> 3) * 256;
        const u32x2 a = read_transposed(from);
        u32x2 b2 = {0u, 0u};
        if constexpr (TILES == 2) b2 = read_transposed(from + 16 * T::PITCH);
        const u32x4 vt = {a[0], a[1], b2[0], b2[1]};
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
    constexpr int CH = DP / 4;  // pieces of 4 values in a row
    constexpr int PASSES = (16 * CH + T::THREADS - 1) / T::THREADS;
    const auto rs = rsrc_of(c.part, gridDim.x * 2u * (uint32_t)(T::PART * 4));
    f32x4 sum[PASSES];
    f32x2 ms[PASSES];
#pragma unroll
    for (int n = 0; n < PASSES; ++n) {
      const int e = n * T::THREADS + (int)threadIdx.x, r = e / CH, ch = e % CH;
      sum[n] = f32x4{0.f, 0.f, 0.f, 0.f}, ms[n] = f32x2{-INFINITY, 0.f};
      if (r >= 16) continue;
#pragma unroll
      for (int w = 0; w < T::WAVES; ++w) ms[n][0] = fmaxf(ms[n][0], ml[w][0][r]);
      const float by = ms[n][0] == -INFINITY ? 0.f : ms[n][0];
#pragma unroll
      for (int w = 0; w < T::WAVES; ++w) {
        const float f = exp2_(ml[w][0][r] - by);
        ms[n][1] = __builtin_fmaf(ml[w][1][r], f, ms[n][1]);
        const f32x4 ow = *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(smem + w * T::WAVE_BYTES) + r * T::O_PITCH + 4 * ch);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[n][i] = __builtin_fmaf(ow[i], f, sum[n][i]);
      }
      if (!p.alone) {
        const uint32_t slot = place_of(me, p.began, T::PART);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sum[n]), rs, (int)(slot + (uint32_t)(r * DP + 4 * ch) * 4u), 0, kDevice);
        if (ch == 0)
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, ms[n]), rs, (int)(slot + (uint32_t)(16 * DP + 2 * r) * 4u), 0, kDevice);
      }
    }
    bool write = true;
    if (!p.alone) {
      const Joining join = joining(c, p, walk.share);
      const int parts = join.parts;
      write = last_of(c, sh, join);
      if (write) {
#pragma unroll 1
        for (int n = 0; n < PASSES; ++n) {
          const int e = n * T::THREADS + (int)threadIdx.x, r = min(e / CH, 15), ch = e % CH;
          f32x4 v4 = {0.f, 0.f, 0.f, 0.f};
          f32x2 t2 = {-INFINITY, 0.f};
#pragma unroll 1
          for (int w0 = 0; w0 < parts; w0 += 8) {
            f32x4 a[8];
            f32x2 t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int w = min(w0 + j, parts - 1);
              const uint32_t slot = place_of(join, w, T::PART);
              a[j] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(slot + (uint32_t)(r * DP + 4 * ch) * 4u), 0, kDevice));
              t[j] = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(slot + (uint32_t)(16 * DP + 2 * r) * 4u), 0, kDevice));
            }
            float now = t2[0];
#pragma unroll
            for (int j = 0; j < 8; ++j) now = fmaxf(now, t[j][0]);
            const float by = now == -INFINITY ? 0.f : now, f0 = exp2_(t2[0] - by);
            t2[0] = now, t2[1] = t2[1] * f0, v4 = v4 * f0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float f = w0 + j < parts ? exp2_(t[j][0] - by) : 0.f;
              if (w0 + j >= parts) continue;
              t2[1] = __builtin_fmaf(t[j][1], f, t2[1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) v4[i] = __builtin_fmaf(a[j][i], f, v4[i]);
            }
          }
          if (PASSES == 1 || n == 0) sum[0] = v4, ms[0] = t2;
          else sum[PASSES - 1] = v4, ms[PASSES - 1] = t2;
        }
      }
    }
    if (write) {
#pragma unroll
      for (int n = 0; n < PASSES; ++n) {
        const int e = n * T::THREADS + (int)threadIdx.x, r = e / CH, ch = e % CH;
        const Row w = row_of(c, p, min(r, 15));
        if (r >= 16 || !w.valid) continue;
        const float total = ms[n][1];
        const bool some = total > 0.f || total != total;
        const float by = some ? 1.f / total : 0.f;
        if (4 * ch < c.D)
          *reinterpret_cast<u32x2 *>(c.out + (size_t)w.token * c.out_row + (size_t)w.head * c.out_head + 4 * ch) =
              u32x2{pack2(sum[n][0] * by, sum[n][1] * by), pack2(sum[n][2] * by, sum[n][3] * by)};
        if (ch == 0 && c.lse != nullptr)
          c.lse[(size_t)w.token * c.Hq + w.head] = some ? (ms[n][0] + __builtin_amdgcn_logf(total)) * kLn2 : -INFINITY;
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ many rows
//
// Chunks of a prompt: 256 rows of tokens times heads that share keys, 32 of each wave, against tiles of keys in a ring of
// four that direct-to-LDS loads fill ahead.  S^T = K Q^T in 32x32x16 MFMAs leaves a lane 16 of 32 keys' scores of one row
// (the other half of the wave has the other 16), which, rounded to bf16, are the second product's operand as they
// lie: O^T = V^T P^T over the keys in that order, values read transposed.  Heads beyond 128 values, whose o and q would
// fill the registers, have 16 rows a wave and 16x16x32 MFMAs (a lane has 4 of 16 keys): every wave reads the tile from LDS for half
// as many rows, and two waves a SIMD fit (a prompt of 4096, heads of 256: 232 us with one wave of 32 rows, 203 so, now 175).  m and l are
// one register a lane, and so is what o has to be scaled by.  The weights' rounding (8 bits) is of the same size as the output's
// own; l sums them unrounded.
// Scaling o costs as much as half of a tile's exponentials: m stays behind the maximum until it would have to grow by
// kSlack, so that weights are up to 2^kSlack and o is scaled once or twice in all.
template <int DP>
struct ManyTile {
  static constexpr int WAVES = 8, THREADS = 64 * WAVES;
  static constexpr int R = DP <= 128 ? 32 : 16;        // rows of a wave, and side of its matrix instructions
  static constexpr int P = 64 / R;                     // parts of a wave, each with a lane for every row
  static constexpr int ROWS = R * WAVES, KEYS = 2 * R;
  static constexpr int STEP = 8 * P;                   // of the products' inner index in an instruction
  static constexpr int KS = DP / STEP, DT = DP / R, KT = 2, WT = KEYS / STEP;
  static constexpr int N = R / P;                      // values of a result tile that a lane has: 4 of every 4 P rows
  typedef float Acc __attribute__((ext_vector_type(N)));
  static constexpr int ROOM = DP == 96 ? 128 : DP;     // values that a row in LDS has room for
  static constexpr int CH = ROOM / 8;                  // 16-byte chunks of a row
  static constexpr int PITCH = ROOM * 2;
  static constexpr int OPERAND = KEYS * PITCH;         // bytes of a tile of K, and of V
  static constexpr int STAGES = 4;                     // of the ring of tiles of K, and of that of V
  static constexpr int ZEROS = OPERAND;                // bytes of zeros behind the rings
  static constexpr int LDS = 2 * STAGES * OPERAND + ZEROS;
  static constexpr int PASS_ROWS = THREADS / CH, PASSES = KEYS / PASS_ROWS;
  static constexpr int DMAS = 2 * PASSES;              // of a wave for a tile
  static constexpr int PART = ROWS * (DP + 2);
  static constexpr int PER_CU = 1;
  static constexpr int IDS = 256;                      // page numbers that a wave has at hand
};
constexpr float kSlack = 8.f;

// Physical chunk of chunk c in row r: a read of K sends 16 rows at one chunk, one of V, by 32 lanes, 4 rows at 4
// chunks in a row.
template <int DP>
__device__ __forceinline__ int many_swizzle_k(int r, int c) {
  if constexpr (ManyTile<DP>::CH >= 16) return c ^ (r & 15);
  else return swz<8>(r, c);
}
template <int DP>
__device__ __forceinline__ int many_swizzle_v(int r, int c) {
  if constexpr (DP > 128) return few_swizzle<DP>(r, c);  // 8 rows at 2 chunks in a row
  else return swz_kn<ManyTile<DP>::CH>(r, c);
}
template <int DP>
__device__ __forceinline__ typename ManyTile<DP>::Acc many_mfma(u32x4 a, u32x4 b, typename ManyTile<DP>::Acc c) {
  if constexpr (ManyTile<DP>::R == 32) return mfma32(a, b, c);
  else return mfma16(a, b, c);
}
// Over the lanes that have a row, the same bits in all of them.
template <int DP>
__device__ __forceinline__ float row_max(float v) {
  if constexpr (ManyTile<DP>::R == 32) return max_halves(v);
  else return max_quarters(v);
}
template <int DP>
__device__ __forceinline__ float row_sum(float v) {
  if constexpr (ManyTile<DP>::R == 32) return sum_halves(v);
  else return sum_quarters(v);
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

// What the workgroup shares beside the tiles.
template <int DP>
struct ManyShared {
  WalkShared<ManyTile<DP>::THREADS> walk;
  int32_t ids[ManyTile<DP>::WAVES][ManyTile<DP>::IDS];
  uint32_t bad_rows[8][2];  // keys of tile b whose page is none: [b % 8]
};

// A wave's loads of an item's tiles: all waves load a part of each.
// FULL: heads of DP values, no fewer.
template <int DP, bool FULL>
struct TileLoads {
  using T = ManyTile<DP>;
  const KeyRows &rows;
  const Piece &p;
  ManyShared<DP> &sh;
  const int32_t *table;
  const uint16_t *k, *v;   // of the item's head
  int D, wave, lane;
  uint32_t lds;            // of the ring
  int32_t *ids;
  int ids_from, plain_until;
  bool some_bad, ever_bad; // whether some page at hand, or of the item so far, is none
  // page and row within it of this thread's keys of the tile that is issued next; where such a row of page 0 is, and how
  // far its values are from there; the keys of the tile before
  int index[T::PASSES], off[T::PASSES], step_pages, step_rows;
  uint64_t base[T::PASSES], to_values, before[T::PASSES];

  __device__ __forceinline__ int row(int i) const { return i * T::PASS_ROWS + (wave * 64 + lane) / T::CH; }
  __device__ __forceinline__ void find(int b) {
#pragma unroll
    for (int i = 0; i < T::PASSES; ++i) {
      const int key = min(p.first + b * T::KEYS + row(i), p.last - 1);
      index[i] = rows.page_of(key), off[i] = key - index[i] * rows.page;
      place(i);
    }
  }
  // A thread's chunks of K and of V are the same ones in all its rows.
  static_assert(T::PASS_ROWS % 16 == 0, "");
  __device__ __forceinline__ int chunk_k() const { return many_swizzle_k<DP>(row(0), lane % T::CH); }
  __device__ __forceinline__ int chunk_v() const { return many_swizzle_v<DP>(row(0), lane % T::CH); }
  __device__ __forceinline__ void place(int i) {
    base[i] = (uint64_t)(size_t)(k + 8 * chunk_k()) + (uint64_t)(uint32_t)off[i] * rows.row_bytes;
  }
  __device__ __forceinline__ void start(int b) {
    step_pages = rows.page_of(T::KEYS), step_rows = T::KEYS - step_pages * rows.page;
    to_values = (uint64_t)(size_t)(v + 8 * chunk_v()) - (uint64_t)(size_t)(k + 8 * chunk_k());
    fill(b), find(b);
  }
  // Rows of the next tile; in pages that a tile is a whole number of they stay (2 to 4 % of a prompt's time).
  __device__ __forceinline__ void advance() {
    if (step_rows == 0) return;
#pragma unroll
    for (int i = 0; i < T::PASSES; ++i) {
      off[i] += step_rows;
      const bool over = off[i] >= rows.page;
      off[i] -= over ? rows.page : 0, index[i] += over ? 1 : 0;
      place(i);
    }
  }
  __device__ __forceinline__ void fill(int b) {  // page numbers from tile b's first on
    ids_from = rows.page_of(p.first + b * T::KEYS);
    const int end = rows.page_of(min(p.first + p.b1 * T::KEYS, p.last) - 1) + 1;
    bool bad = false;
#pragma unroll 1
    for (int i = lane; i < T::IDS; i += 64)
      if (ids_from + i < end) {
        const int id = table[ids_from + i];
        ids[i] = id;
        bad = bad || rows.bad(id);
      }
    some_bad = __ballot(bad) != 0;
    asm volatile("" ::: "memory");  // the wave's LDS accesses are served in order
    // whole tiles, and those whose page numbers are at hand
    const int64_t known = (int64_t)(ids_from + T::IDS) * rows.page - p.first;
    plain_until = some_bad ? 0 : (int)(min((int64_t)(p.last - p.first), known) / T::KEYS);
  }
  // What the loads of tiles from plain_until on need beside the others': where keys lie, if the tile is not whole (or past
  // the last one), page numbers that are not at hand, a note of pages that are none.
  __device__ __forceinline__ void prepare(int b) {
    asm volatile("" : "+s"(b));  // a branch: none of this is made for the others
    const int end = p.first + (b + 1) * T::KEYS;
    if (end > p.last) find(b);
    if (rows.page_of(min(end, p.last) - 1) >= ids_from + T::IDS) fill(b);
    if (some_bad) {
      ever_bad = true;
#pragma unroll
      for (int i = 0; i < T::PASSES; ++i)
        if (rows.bad(ids[index[i] - ids_from]) && lane % T::CH == 0) atomicOr(&sh.bad_rows[b % 8][row(i) >> 5], 1u << (row(i) & 31));
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): there for the barrier
    }
  }
  // The page numbers of tile b, then the loads of its keys and of the values of the tile before, which are on their way after
  // this; what the stages held has been read.  Past the last tile the last key is loaded, which nobody reads: every wave has
  // as many loads in every interval.
  __device__ __forceinline__ void pages(int (&id)[T::PASSES]) const {
#pragma unroll
    for (int i = 0; i < T::PASSES; ++i) id[i] = ids[index[i] - ids_from];
  }
  __device__ __forceinline__ void issue(int b, const int (&id)[T::PASSES], bool values = true) {
    const uint32_t to = lds + (uint32_t)wave * 1024u;
    const uint32_t to_k = to + (uint32_t)(b % T::STAGES) * T::OPERAND, to_v = to + (uint32_t)(T::STAGES + (b - 1 + T::STAGES) % T::STAGES) * T::OPERAND;
#pragma unroll
    for (int i = 0; i < T::PASSES; ++i) {
      const uint64_t at = (uint64_t)(rows.bad(id[i]) ? 0u : (uint32_t)id[i]) * rows.page_bytes + base[i];
      if (FULL || 8 * chunk_k() < D) global_dma16(reinterpret_cast<const void *>(at), to_k + (uint32_t)(i * T::THREADS * 16));
      if (values && (FULL || 8 * chunk_v() < D))
        global_dma16(reinterpret_cast<const void *>(before[i] + to_values), to_v + (uint32_t)(i * T::THREADS * 16));
      before[i] = at;
      index[i] += step_pages;
    }
  }
  __device__ __forceinline__ void all(int b, bool values = true) {
    int id[T::PASSES];
    if (b >= plain_until) prepare(b);
    pages(id);
    issue(b, id, values);
    advance();
  }
};

// The operands' fragments as a wave reads them from a tile.
template <int DP>
struct Fragments {
  using T = ManyTile<DP>;
  uint32_t k0, v0, vt0;
  __device__ __forceinline__ Fragments(uint32_t lds, int lane) {
    const int row = lane % T::R, part = lane / T::R, l16 = lane & 15, r = 4 * part + (l16 >> 2);
    k0 = lds + (uint32_t)(row * T::PITCH + many_swizzle_k<DP>(row, part) * 16);
    vt0 = lds + T::STAGES * T::OPERAND;
    v0 = vt0 + r * T::PITCH + many_swizzle_v<DP>(r, 2 * (row >> 4) + ((l16 & 3) >> 1)) * 16 + 8 * (l16 & 1);
  }
  // Key R t + l % R, values STEP s + 8 (l / R) .. + 7.
  __device__ __forceinline__ void keys(int b, int t, u32x4 (&k)[T::KS]) const {
    constexpr int IN = 16 / T::P;  // steps in 256 bytes
    const uint32_t from = k0 + stage(b);
#pragma unroll
    for (int s = 0; s < T::KS; ++s)
      k[s] = *(__attribute__((address_space(3))) const u32x4 *)(size_t)((from ^ ((s % IN) * 16 * T::P)) + (s / IN) * 256 + T::R * t * T::PITCH);
  }
  // Values R (t0 + t) + l % R of the 8 keys of STEP s .. that the lane's weights are of.
  __device__ __forceinline__ uint32_t stage(int b) const { return (uint32_t)(b % T::STAGES) * T::OPERAND; }
  template <int N>
  __device__ __forceinline__ void values(uint32_t stage, int t0, u32x4 (&v)[N][T::WT]) const {
    constexpr int IN = 128 / T::R;  // tiles of values in 256 bytes
    const uint32_t from = v0 + stage;
#pragma unroll
    for (int s = 0; s < T::WT; ++s)  // in the order in which multiply() uses them
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const uint32_t at = (from ^ (((t0 + t) % IN) * 2 * T::R)) + ((t0 + t) / IN) * 256;
        const u32x2 a = read_transposed(at + T::STEP * s * T::PITCH), b2 = read_transposed(at + (T::STEP * s + 4 * T::P) * T::PITCH);
        v[t][s] = u32x4{a[0], a[1], b2[0], b2[1]};
      }
  }
};

// A wave's rows, their running maximum and sum (in powers of 2) and o.
template <int DP>
struct RowState {
  using T = ManyTile<DP>;
  using Acc = typename T::Acc;
  Acc acc[T::DT];
  float m, l;
  int large;  // large_maximum of the rows' m
  __device__ __forceinline__ void clear() {
    m = -INFINITY, l = 0.f, large = 0;
#pragma unroll
    for (int t = 0; t < T::DT; ++t)
#pragma unroll
      for (int i = 0; i < T::N; ++i) acc[t][i] = 0.f;
  }
  // Scores of the keys from kb on (tile b) to weights.  `masked`: not all are seen by all rows.  True if there are
  // infinities or NaN among such a tile's values: they must not reach rows that do not see them, and have gone into o
  // one by one.
  __device__ __forceinline__ bool weigh(Acc (&x)[T::KT], u32x4 (&w)[T::WT], float scale, bool masked, int b, int kb, const Row &row,
                                        uint32_t bad0, uint32_t bad1, const Fragments<DP> &from, int lane) {
    const int part = lane / T::R;
    const uint32_t vt0 = from.vt0 + from.stage(b);
    bool odd = false;
    if (masked) {
      // a lane's scores are of keys R t + 4 P (i / 4) + 4 part + i % 4
      const int lo = row.lo - kb - 4 * part, hi = row.hi - kb - 4 * part;
#pragma unroll
      for (int t = 0; t < T::KT; ++t) {
        const uint32_t bad = (T::R * t >= 32 ? bad1 : bad0) >> (T::R * t % 32 + 4 * part);
#pragma unroll
        for (int i = 0; i < T::N; ++i) {
          const int at = 4 * T::P * (i >> 2) + (i & 3);
          x[t][i] = T::R * t + at >= lo && T::R * t + at < hi && !((bad >> at) & 1u) ? x[t][i] : -INFINITY;
        }
      }
      uint32_t bits = 0;
#pragma unroll 4
      for (int i = 0; i < T::OPERAND / 1024; ++i) {
        const u32x4 four = *(__attribute__((address_space(3))) const u32x4 *)(size_t)(vt0 + (uint32_t)(i * 64 + lane) * 16u);
#pragma unroll
        for (int j = 0; j < 4; ++j) bits |= pair_exponents(four[j]);
      }
      odd = __ballot((bits & 0x80008000u) != 0) != 0;
    }
    float top = x[0][0];
#pragma unroll
    for (int i = 1; i < T::N * T::KT; ++i) top = fmaxf(top, x[i / T::N][i % T::N]);
    top = row_max<DP>(top) * scale;
    const bool grows = top > m + kSlack;
    if (__ballot(grows) != 0) {
      // each row by itself: its bits do not depend on the others', nor on keys that only they see
      const float now = grows ? top : m, less = grows ? exp2_(m - now) : 1.f;
      m = now;
      large = uniform(large_maximum(m) ? 1 : 0);
      l = l * less;
#pragma unroll
      for (int t = 0; t < T::DT; ++t) acc[t] = acc[t] * less;
    }
    if (odd) {
#pragma unroll 1
      for (int r = 0; r < T::KEYS; ++r) {
        const bool seen = kb + r >= row.lo && kb + r < row.hi && !(((r & 32 ? bad1 : bad0) >> (r & 31)) & 1u);
#pragma unroll
        for (int t = 0; t < T::DT; ++t)
#pragma unroll
          for (int i = 0; i < T::N / 4; ++i) {
            // values R t + 4 P i + 4 part .. + 3 of key r
            const uint32_t a = vt0 + r * T::PITCH + many_swizzle_v<DP>(r, (T::R * t + 4 * T::P * i + 4 * part) >> 3) * 16 + 8 * (part & 1);
            const u32x2 h = *(__attribute__((address_space(3))) const u32x2 *)(size_t)a;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t f = (h[j >> 1] >> (16 * (j & 1))) & 0xFFFFu;
              if (seen && (f & 0x7F80u) == 0x7F80u) acc[t][4 * i + j] = acc[t][4 * i + j] + as_float(f << 16);
            }
          }
      }
    }
    float by = m == -INFINITY ? 0.f : m;
    if (large != 0) exact_maximum(x, scale, by);
#pragma unroll
    for (int t = 0; t < T::KT; ++t)
#pragma unroll
      for (int i = 0; i < T::N; i += 2) {
        const float e0 = exp2_(__builtin_fmaf(x[t][i], scale, -by)), e1 = exp2_(__builtin_fmaf(x[t][i + 1], scale, -by));
        l = l + (e0 + e1);
        w[(T::N * t + i) / 8][(T::N * t + i) % 8 / 2] = pack2(e0, e1);
      }
    return odd;
  }
  // Infinities and NaN that weigh() has seen to, out of the values.
  template <int N>
  __device__ __forceinline__ static void only_finite(u32x4 (&v)[N][T::WT]) {
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int s = 0; s < T::WT; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[t][s][i] = pair_finite(v[t][s][i]);
  }
  // o of the values R t0 and on.
  template <int N>
  __device__ __forceinline__ void multiply(const u32x4 (&v)[N][T::WT], const u32x4 (&w)[T::WT], int t0) {
#pragma unroll
    for (int s = 0; s < T::WT; ++s)
#pragma unroll
      for (int t = 0; t < N; ++t) acc[t0 + t] = many_mfma<DP>(v[t][s], w[s], acc[t0 + t]);
  }

  // The item's part is whole: to the output, or beside the others' and, if it is the last of them, joined, always in the
  // parts' order.  A partial result lies as the lanes have it, 1 KB an instruction.
  __device__ __forceinline__ void finish(const AttnCall &c, WalkShared<T::THREADS> &sh, const Piece &p, const AttnShare &share, const Row &row,
                                         int me, int wave, int lane) {
    const auto rs = rsrc_of(c.part, gridDim.x * 2u * (uint32_t)(T::PART * 4));
    const int r = wave * T::R + lane % T::R, part = lane / T::R;
    l = row_sum<DP>(l);
    bool write = true;
    if (!p.alone) {
      const uint32_t at = (uint32_t)(wave * T::R * DP * 4 + lane * 16), at_sums = (uint32_t)(T::ROWS * DP + 2 * r) * 4u;
      const Joining join = joining(c, p, share);
      write = others_done(c, sh, join);
      if (!write) {
        const uint32_t slot = place_of(me, p.began, T::PART);
#pragma unroll
        for (int t = 0; t < T::DT; ++t)
#pragma unroll
          for (int i = 0; i < T::N / 4; ++i) {
            const f32x4 v = {acc[t][4 * i], acc[t][4 * i + 1], acc[t][4 * i + 2], acc[t][4 * i + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, (int)(slot + at + (uint32_t)(T::N / 4 * t + i) * 1024u), 0, kDevice);
          }
        if (part == 0)
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{m, l}), rs, (int)(slot + at_sums), 0, kDevice);
        write = last_of(c, sh, join);
      }
      if (write) {
        const RowState own = *this;
        clear();
#pragma unroll 1
        for (int s = 0; s < join.parts; ++s) {
          constexpr int ONCE = T::DT < 4 ? T::DT : 4, Q = T::N / 4;  // so that loads and sums fit into the registers
          const bool mine = join.counter + s == me;
          const uint32_t slot = place_of(join, s, T::PART);
          f32x2 sums = {own.m, own.l};
          if (!mine) sums = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(slot + at_sums), 0, kDevice));
          float f0 = 0.f, f1 = 0.f;
#pragma unroll
          for (int t0 = 0; t0 < T::DT; t0 += ONCE) {
            f32x4 v[ONCE][Q];
#pragma unroll
            for (int t = 0; t < ONCE; ++t)
#pragma unroll
              for (int i = 0; i < Q; ++i) {
                const Acc &o = own.acc[t0 + t];
                v[t][i] = f32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
              }
            if (!mine) {
#pragma unroll
              for (int t = 0; t < ONCE; ++t)
#pragma unroll
                for (int i = 0; i < Q; ++i)
                  v[t][i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(slot + at + (uint32_t)(Q * (t0 + t) + i) * 1024u), 0, kDevice));
            }
            if (t0 == 0) {
              const float now = fmaxf(m, sums[0]), by = now == -INFINITY ? 0.f : now;
              f0 = exp2_(m - by), f1 = exp2_(sums[0] - by);
              m = now;
              l = __builtin_fmaf(sums[1], f1, l * f0);
            }
#pragma unroll
            for (int t = 0; t < ONCE; ++t)
#pragma unroll
              for (int i = 0; i < T::N; ++i) acc[t0 + t][i] = __builtin_fmaf(v[t][i >> 2][i & 3], f1, acc[t0 + t][i] * f0);
          }
        }
      }
    }
    if (write && row.valid) {
      const bool some = l > 0.f || l != l;
      const float by = some ? 1.f / l : 0.f;
      uint16_t *to = c.out + (size_t)row.token * c.out_row + (size_t)row.head * c.out_head;
#pragma unroll
      for (int t = 0; t < T::DT; ++t)
#pragma unroll
        for (int i = 0; i < T::N / 4; ++i) {
          const int d = T::R * t + 4 * T::P * i + 4 * part;
          if (d < c.D)
            *reinterpret_cast<u32x2 *>(to + d) = u32x2{pack2(acc[t][4 * i] * by, acc[t][4 * i + 1] * by),
                                                       pack2(acc[t][4 * i + 2] * by, acc[t][4 * i + 3] * by)};
        }
      if (part == 0 && c.lse != nullptr)
        c.lse[(size_t)row.token * c.Hq + row.head] = some ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    }
  }
};

// The schedule of what precedes: N matrix instructions, each followed by reads of LDS and vector instructions.
template <int N, int READS, int VALU>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    if constexpr (VALU > 0) __builtin_amdgcn_sched_group_barrier(0x002, VALU, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Two waves share a SIMD, one of waves 0-3 and one of waves 4-7, and take turns at the matrix pipe: each makes a tile's
// weights and then multiplies (o of the tile, then the scores of the next one: 32 MFMAs, 1024 cycles, with heads of 128), and one
// barrier a tile, which waves 0-3 have after multiplying and waves 4-7 after the weights, keeps them half a tile apart.
//   In interval b, between two barriers, waves 0-3 make weights of tile b and o of it and scores of b + 1, waves 4-7 o of
// b - 1, scores of b and weights of b: keys of b and b + 1 are read, values of b - 1 and b.  All ask for keys of
// b + 3 and values of b + 2, whose stages (of b - 1 and b - 2) nobody reads, in the time that the matrix instructions
// leave, and before the barrier wait for what they asked for in the interval before: it is read from the next on.
//   A causal prompt of 8192, 32 heads over 8 of 128: 505 to 547 us, 1000 to 1085 TFLOP/s.  The matrix pipes are 56 % busy (LDS 29 %,
// no bank conflicts), a tile takes about 3300 cycles for two waves' 2086 of products, at a clock that the board's power
// lowers from 2.1 to 1.8 GHz (2.2 on constant operands); without exponentials it takes 9 % fewer cycles, without loads to LDS 12,
// without reads of LDS 12.  With four waves of 32 rows, one a SIMD, it took 722 us, with two barriers a tile 523.  Heads of 64: half
// the products, as many exponentials: 325 to 360 us, pipes 37 % busy.  128 tokens over 30000 keys, 32 heads over 4 of 256: 152 us,
// 830 TFLOP/s.
template <int DP, bool FULL>
__global__ __launch_bounds__(ManyTile<DP>::THREADS, ManyTile<DP>::PER_CU) void attn_pairs_kernel(AttnCall c) {
  using T = ManyTile<DP>;
  constexpr int KS = T::KS, DT = T::DT, KT = T::KT, WT = T::WT;
  extern __shared__ __align__(256) unsigned char ring[];
  __shared__ ManyShared<DP> sh;
  const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), part = lane / T::R;
  const bool behind = wave >= 4;
  const uint32_t lds = lds_address(ring);
  const KeyRows rows(c);
  const float scale = own_register(c.scale);
  const Fragments<DP> from(lds, lane);
  const int me = (int)xcd_remap(blockIdx.x, gridDim.x);

  // chunks that the heads do not have stay zero, and what lies behind the ring
  for (int i = (FULL ? 2 * T::STAGES * T::OPERAND / 16 : 0) + threadIdx.x; i < T::LDS / 16; i += T::THREADS)
    reinterpret_cast<u32x4 *>(ring)[i] = u32x4{0u, 0u, 0u, 0u};
  auto barrier = [&]() {  // nothing moves across it
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };

  Walk<T::THREADS, false> walk(c, sh.walk, me, (int)gridDim.x);
#pragma unroll 1
  for (; walk.next(); walk.done()) {
    const Piece &p = walk.p;
    const Row row = row_of(c, p, wave * T::R + lane % T::R);
    const auto [all_lo, all_hi] = attn_all_see(c.cut, p.s, p.tile, c.by_heads(wave * T::R), c.by_heads(wave * T::R + T::R - 1) + 1);
    // tiles whose keys all rows see
    const int clear_from = uniform((max(all_lo - p.first, 0) + T::KEYS - 1) / T::KEYS), clear_to = uniform(max(all_hi - p.first, 0) / T::KEYS);
    TileLoads<DP, FULL> loads{rows, p, sh, c.table + (size_t)p.request * c.table_pitch, c.k + (size_t)p.kv * c.cache_head,
                              c.v + (size_t)p.kv * c.cache_head, c.D, wave, lane, lds, sh.ids[wave]};
    loads.ever_bad = false;
    if (threadIdx.x < 16) (&sh.bad_rows[0][0])[threadIdx.x] = 0u;
    u32x4 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = u32x4{0u, 0u, 0u, 0u};
      if (row.valid && (FULL || T::STEP * s + 8 * part < c.D))
        q[s] = *reinterpret_cast<const u32x4 *>(c.q + (size_t)row.token * c.q_row + (size_t)row.head * c.q_head + T::STEP * s + 8 * part);
    }
    if (p.b0 < p.b1) loads.start(p.b0);
    RowState<DP> state;
    state.clear();
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): from here on only direct loads to LDS are counted
    __syncthreads();
    if (p.b0 < p.b1) {
      for (int i = 0; i < 3; ++i) loads.all(p.b0 + i, i > 0);
      wait_vmcnt<2 * T::DMAS>();
      barrier();
      typename T::Acc x[KT];
      auto score = [&](const u32x4 (&k)[KS], typename T::Acc &to) {
#pragma unroll
        for (int i = 0; i < T::N; ++i) to[i] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) to = many_mfma<DP>(k[s], q[s], to);
      };
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        u32x4 k[KS];
        from.keys(p.b0, t, k);
        score(k, x[t]);
      }
      wait_vmcnt<T::DMAS>();
      barrier();
      if (behind) loads.all(p.b0 + 3);
      const int ahead = behind ? 4 : 3;
#pragma unroll 1
      for (int b = p.b0; b < p.b1; ++b) {
        // weigh.  The wave that multiplies goes first: the other's instructions fill what it leaves (712 -> 693 us for a prompt
        // of 8192, together with the values' order).
        __builtin_amdgcn_s_setprio(0);
        u32x4 v0[DT - DT / 2][WT], v1[DT / 2][WT], w[WT];
        uint32_t bad0 = 0, bad1 = 0;
        if (loads.ever_bad) {
          bad0 = sh.bad_rows[b % 8][0], bad1 = sh.bad_rows[b % 8][1];
          if (threadIdx.x < 2) sh.bad_rows[(b + T::STAGES) % 8][threadIdx.x] = 0u;
        }
        const int kb = p.first + b * T::KEYS;
        const bool masked = b < clear_from || b >= clear_to || loads.ever_bad;
        uint32_t stage = from.stage(b);
        const int odd = uniform(state.weigh(x, w, scale, masked, b, kb, row, bad0, bad1, from, lane) ? 1 : 0);
#pragma unroll
        for (int s = 0; s < WT; ++s) asm volatile("" : "+v"(w[s]), "+v"(state.l));  // made here: the scores' registers are free
        if (odd != 0) {
          // o of this tile here and now; the products that are to come add zeros
#pragma unroll
          for (int t = 0; t < DT; ++t) {
            u32x4 v[1][WT];
            from.values(stage, t, v);
            RowState<DP>::only_finite(v);
            state.multiply(v, w, t);
          }
#pragma unroll
          for (int s = 0; s < WT; ++s) w[s] = u32x4{0u, 0u, 0u, 0u};
          stage = T::STAGES * T::OPERAND;  // where zeros are, as a tile's values
        }
        __builtin_amdgcn_sched_barrier(0);
        from.values(stage, 0, v0);
        if (behind) wait_vmcnt<T::DMAS>(), barrier();
        // multiply: o, then the next tile's scores (past the last tile they are not used).  Each part's operands are read
        // while the part before runs: no more than two at a time have registers.
        __builtin_amdgcn_s_setprio(1);
        if (b + ahead >= loads.plain_until) loads.prepare(b + ahead);
        int id[T::PASSES];
        u32x4 k0[KS], k1[KS];
        constexpr int SECOND = DT / 2 * WT;  // matrix instructions of o's second part
        loads.pages(id);
        from.values(stage, DT - DT / 2, v1);
        state.multiply(v0, w, 0);
        interleave<DT * WT - SECOND, 2, 0>();
        from.keys(b + 1, 0, k0);
        loads.issue(b + ahead, id);
        state.multiply(v1, w, DT - DT / 2);
        interleave<SECOND, (KS + SECOND - 1) / SECOND, 6>();
        from.keys(b + 1, 1, k1);
        score(k0, x[0]);
        interleave<KS, 1, 0>();
        score(k1, x[1]);
        if (!behind) wait_vmcnt<T::DMAS>(), barrier();
        loads.advance();
      }
      __builtin_amdgcn_s_setprio(0);
    }
    state.finish(c, sh.walk, p, walk.share, row, me, wave, lane);
    __syncthreads();
  }
}

// ------------------------------------------------------------------ launches

int padded_head(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

template <int DP, bool MANY, bool FULL>
int launch(const AttnCall &c, int grid, hipStream_t s) {
  void (*fn)(AttnCall);
  if constexpr (MANY) fn = attn_pairs_kernel<DP, FULL>;
  else fn = attn_few_kernel<DP>;
  constexpr int lds = MANY ? ManyTile<DP>::LDS : FewTile<DP>::WAVES * FewTile<DP>::WAVE_BYTES;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return OCC_ENODEV;
  static Once limit_set[kMaxDevices];
  if (!limit_set[dev].run([&] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
      }))
    return OCC_EHIP;
  hipLaunchKernelGGL(fn, dim3(grid), dim3(MANY ? ManyTile<DP>::THREADS : FewTile<DP>::THREADS), lds, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}
template <int DP, bool MANY>
int launch(const AttnCall &c, int grid, hipStream_t s) {
  // tiles of rows as wide as 128 values, products of 96 (a prompt of 4096, 32 heads over 8 of 80: 126 us, 142 with products of 128)
  if (MANY && DP == 128 && c.D <= 96) return launch<96, true, false>(c, grid, s);
  return MANY && c.D == DP ? launch<DP, MANY, true>(c, grid, s) : launch<DP, MANY, false>(c, grid, s);
}
template <bool MANY>
int launch(const AttnCall &c, int DP, int grid, hipStream_t s) {
  return DP == 64 ? launch<64, MANY>(c, grid, s) : DP == 128 ? launch<128, MANY>(c, grid, s) : launch<256, MANY>(c, grid, s);
}

constexpr int kJoined = kCus;  // counters, a workgroup
int many_rows(int DP) { return DP > 128 ? ManyTile<256>::ROWS : ManyTile<128>::ROWS; }
int many_keys(int DP) { return DP > 128 ? ManyTile<256>::KEYS : ManyTile<128>::KEYS; }
int few_keys(int DP) { return DP > 128 ? FewTile<256>::KEYS : FewTile<128>::KEYS; }

}  // namespace

size_t attn_workspace(int D) {
  const int DP = padded_head(D);
  // two partial results a workgroup, one workgroup a CU; those of many rows are the larger
  return (size_t)kJoined * 4 + (size_t)kCus * 2 * many_rows(DP) * (DP + 2) * 4;
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
  c.page_bytes = (uint32_t)a.cache_page * 2u, c.row_bytes = (uint32_t)a.cache_row * 2u, c.cache_head = a.cache_head;
  c.scale = a.scale * kLog2e;
  c.joined = static_cast<uint32_t *>(a.workspace);
  c.part = reinterpret_cast<float *>(static_cast<unsigned char *>(a.workspace) + (size_t)kJoined * 4);
  const int DP = padded_head(a.D), cus = std::min(di->num_cus, kCus);
  auto go = [&](bool many, int least, int most) {
    AttnCall k = c;
    const int rows = many ? many_rows(DP) : FewTile<128>::ROWS;
    k.heads = std::min(c.group, rows);
    k.cut.tokens = rows / k.heads, k.cut.by_tokens = Divider(k.cut.tokens);
    k.groups = (c.group + k.heads - 1) / k.heads;
    k.by_heads = Divider(k.heads), k.by_groups = Divider(k.groups);
    k.cut.parts = a.Hkv * k.groups;
    // Keys' worth of an item's beginning and end.  Many rows: 11 us (a piece's q, pages and first tiles, a masked tile, its
    // output), a tile of 64 keys 1.8 us; with 128 in place of 512 a prompt of 8192 took 682 us instead of 565, whose short
    // items fell to few workgroups, and with 1024 570.  Heads of 256: 384 (prompts of 4096 and 8192 212 and 354 us, with 256 231 and
    // 383, with 768 217 and 361).  Few rows: 128 and 512 make 64 requests 1 % slower.
    k.cut.fixed = many ? (DP <= 128 ? 512 : 384) : 256, k.cut.block = many ? many_keys(DP) : few_keys(DP);
    k.cut.window = a.window < c.keys ? a.window : 0, k.cut.causal = a.causal != 0;
    k.least = least, k.most = most;
    // (four chunks of 256 tokens: 57 us with 512 spare, 43 with 1024; four requests of 100 to 900 keys 13.0 us with parts of
    // 128 keys or more, 14.6 with 256, 17.8 with 512; one of 4000 keys 16.6, 16.4, 17.8, but 18.1 with 64;
    // many rows, a prompt of 1024: 32.0 with 256, 33.2 with 512)
    k.min_share = 256, k.least_even = many ? 256 : 128, k.spare = many ? 1024 : 512;
    return many ? launch<true>(k, DP, cus, s) : launch<false>(k, DP, cus, s);
  };
  const int most_rows = (int)std::min<int64_t>((int64_t)std::min(a.max_fresh, a.rows) * c.group, INT32_MAX);
  if (most_rows <= kFewRows) return go(false, 0, INT32_MAX);
  // all requests of the largest size, as far as the host can know
  if (a.requests == 1 || (int64_t)a.requests * a.max_fresh == a.rows) return go(true, 0, INT32_MAX);
  const int few = go(false, 0, kFewRows);
  return few == OCC_OK ? go(true, kFewRows + 1, INT32_MAX) : few;
}

}  // namespace occ
