// What a paged cache needs before its attention: block tables and slots from lengths (occ_kv_tables), rotary positions
// with keys and values put into the cache (occ_rope).
#include "block_util.h"
#include "divider.h"
#include "rope_plan.h"

#include <algorithm>

namespace occ {
namespace {

constexpr int kThreads = 256, kWaves = 4;

// ------------------------------------------------------------------ tables
//
// All sums are over requests: tokens, pages to get, pages that go back.  One launch: every workgroup makes the sums of all
// requests for itself (8 bytes a request from the L2) and then does its share of the requests (pages) and of the tokens.
// Pages come from the ring's head and go back behind its tail, so nothing that one workgroup reads is written by another.
// What bounds it is latency: 64 requests 6.2 us, of which a launch is 2.3 (8.2 with sums through LDS lane by lane, requests
// read again for each pass and twice the code, which is fetched cold); 1500 requests with 360000 tokens 13.
struct TablesCall {
  int n, T, width, pages, size;
  int64_t keys;              // width * page
  Divider by_page;
  int page;
  const int32_t *cached, *fresh, *free;
  int32_t *table, *ring;
  size_t ld;
  int32_t *lens, *starts, *slots, *positions, *free_after;
  int requests, each;        // of a workgroup, tokens of a thread
};

// A request by itself: its tokens, its pages before and after, whether it is over.
struct Asked {
  int64_t tokens;  // 0 for one that is over
  int have, need, back;
  bool fits;       // into its row of the table
};
__device__ __forceinline__ Asked asked(const TablesCall &c, int cached, int fresh) {
  Asked a;
  a.tokens = fresh < 0 ? 0 : fresh;
  const int64_t total = (int64_t)cached + a.tokens;
  a.fits = fresh >= 0 && cached >= 0 && total <= c.keys;
  const int known = (int)min((int64_t)max(cached, 0), c.keys);
  // (x + page - 1) / page without passing 2^31
  a.have = known == 0 ? 0 : c.by_page(known - 1) + 1;
  a.need = a.fits ? (total == 0 ? 0 : c.by_page((int)total - 1) + 1) - a.have : 0;
  a.back = fresh < 0 ? a.have : 0;
  return a;
}

// What requests before one have asked for.
struct Before {
  int64_t tokens, need, back;
};
// `need` counts only for requests whose tokens fit into the step's buffers.
__device__ __forceinline__ bool within(const TablesCall &c, const Asked &a, const Before &b) {
  return a.fits && b.tokens + a.tokens <= c.T;
}
__device__ __forceinline__ void pass(const TablesCall &c, Before &b, const Asked &a) {
  if (within(c, a, b)) b.need += a.need;
  b.tokens += a.tokens;
  b.back += a.back;
}

// STAGED: up to kStaged requests lie in LDS, with what those before them have asked for, so that the passes over them and
// the search for a token's request wait for nothing but LDS.  Beyond, every workgroup reads them from memory for each pass, in
// pieces that a thread takes one by one: single tokens of 2048 requests 12 us, of 2049 14, of 5000 25, of 16384 92, of 65536 930.
constexpr int kStaged = 2048;

template <bool STAGED>
__global__ __launch_bounds__(kThreads) void kv_tables_kernel(TablesCall c) {
  __shared__ int64_t sums[3][kWaves];
  __shared__ Before before[kThreads + 1];   // of each thread's requests
  struct Share {
    int64_t first;  // its first page's place behind the ring's head, or behind its tail
    int have, need, back;
  };
  __shared__ Share shares[64];
  __shared__ int lds_cached[STAGED ? kStaged : 1], lds_fresh[STAGED ? kStaged : 1];
  __shared__ int lds_start[STAGED ? kStaged + 1 : 1], lds_need[STAGED ? kStaged : 1];  // sums before; what passes 31 bits cut
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (c.n + kThreads - 1) / kThreads;
  const int r0 = min((int)threadIdx.x * per, c.n), r1 = min(r0 + per, c.n);
  const int size = c.size;
  const int given[2] = {c.free[0], c.free[1]};
  if constexpr (STAGED) {
    for (int i = threadIdx.x; i < c.n; i += kThreads) lds_cached[i] = c.cached[i], lds_fresh[i] = c.fresh[i];
    __syncthreads();
  }
  const int count = min(max(given[1], 0), size);
  const int head = given[0] < 0 || given[0] >= size ? 0 : given[0];
  auto cached_of = [&](int i) { return STAGED ? lds_cached[i] : c.cached[i]; };
  auto fresh_of = [&](int i) { return STAGED ? lds_fresh[i] : c.fresh[i]; };
  auto short31 = [](int64_t v) { return (int)min(v, (int64_t)0x7FFFFFFF); };

  // Sums before each thread's requests: tokens first, for which requests need pages depends on them.
  auto within_wave = [&](int64_t own, int which) {
    const int64_t upto = sum_upto(own);
    if (lane == 63) sums[which][wave] = upto;
    return upto - own;
  };
  auto waves_before = [&](int which) {
    int64_t sum = 0;
    for (int w = 0; w < wave; ++w) sum += sums[which][w];
    return sum;
  };
  Before own{0, 0, 0};
  for (int i = r0; i < r1; ++i) own.tokens += max(fresh_of(i), 0);
  Before b{within_wave(own.tokens, 0), 0, 0};
  __syncthreads();
  b.tokens += waves_before(0);
  Before mine = b;
  for (int i = r0; i < r1; ++i) pass(c, mine, asked(c, cached_of(i), fresh_of(i)));
  own = mine;
  b.need = within_wave(own.need, 1);
  b.back = within_wave(own.back, 2);
  __syncthreads();
  b.need += waves_before(1);
  b.back += waves_before(2);
  before[threadIdx.x] = b;
  if (threadIdx.x == kThreads - 1) before[kThreads] = Before{own.tokens, b.need + own.need, b.back + own.back};

  // the workgroup's requests: lengths, and what their pages need
  const int first = min((int)blockIdx.x * c.requests, c.n), last = min(first + c.requests, c.n);
  __shared__ int64_t taken;   // pages: the sum up to the last request that gets its own
  if (threadIdx.x == 0) taken = 0;
  __syncthreads();
  {
    Before at = b;
    int64_t most = 0;
    for (int i = r0; i < r1; ++i) {
      const Asked a = asked(c, cached_of(i), fresh_of(i));
      const bool room = at.need + a.need <= count, ok = within(c, a, at) && (a.need == 0 || room);
      if (ok && a.need > 0) most = at.need + a.need;
      if (i >= first && i < last) {
        c.lens[i] = fresh_of(i) < 0 ? 0 : ok ? (int)(cached_of(i) + a.tokens) : -1;
        c.starts[i] = (int)min(at.tokens, (int64_t)c.T);
        if (i == c.n - 1) c.starts[c.n] = (int)min(at.tokens + a.tokens, (int64_t)c.T);
        shares[i - first] = Share{a.back ? at.back : at.need, a.have, ok ? a.need : 0, a.back};
      }
      if constexpr (STAGED) lds_start[i] = short31(at.tokens), lds_need[i] = short31(at.need);
      pass(c, at, a);
    }
    if (blockIdx.x == 0 && most > 0) atomicMax(reinterpret_cast<long long *>(&taken), (long long)most);
  }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int64_t next = head + taken, back = before[kThreads].back;
    if (c.n == 0) c.starts[0] = 0;
    c.free_after[0] = (int)(next < size ? next : next - size);
    c.free_after[1] = (int)min(count - taken + back, size - taken);
  }

  // the workgroup's tokens, c.each that follow each other a thread
  const int64_t all = before[kThreads].tokens;
  const int64_t base = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * c.each, end = min(base + c.each, (int64_t)c.T);
  if (base < end) {
    // the last request that begins at or before the first: of several that begin there, the others have no tokens
    int i = 0;
    Before at{0, 0, 0};
    if (base < all) {
      int lo = 0, hi = STAGED ? c.n - 1 : kThreads - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((STAGED ? (int64_t)lds_start[mid] : before[mid].tokens) <= base) lo = mid;
        else hi = mid - 1;
      }
      i = lo;
      // threads behind the requests' end begin at the sum of all, which is past any token
      if constexpr (!STAGED) at = before[lo], i = lo * per;
    }
#pragma unroll 1
    for (int64_t t = base; t < end; ++t) {
      int slot = -1, position = 0;
      if (t < all) {
        Asked a;
        if constexpr (STAGED) {
          while (i + 1 < c.n && lds_start[i + 1] <= t) ++i;
          a = asked(c, lds_cached[i], lds_fresh[i]);
          at = Before{lds_start[i], lds_need[i], 0};
        } else {
          a = asked(c, c.cached[i], c.fresh[i]);
          while (at.tokens + a.tokens <= t) {
            pass(c, at, a);
            ++i;
            a = asked(c, c.cached[i], c.fresh[i]);
          }
        }
        if (within(c, a, at) && (a.need == 0 || at.need + a.need <= count)) {
          position = cached_of(i) + (int)(t - at.tokens);
          const int index = c.by_page(position);
          const int64_t from = head + at.need + (index - a.have);
          const int id = *(index < a.have ? c.table + (size_t)i * c.ld + index : c.ring + (from < size ? from : from - size));
          if ((uint32_t)id < (uint32_t)c.pages) slot = id * c.page + (position - index * c.page);
        }
      }
      c.slots[t] = slot;
      c.positions[t] = position;
    }
  }
  // and its pages
  for (int i = first + wave; i < last; i += kWaves) {
    const Share s = shares[i - first];
    int32_t *row = c.table + (size_t)i * c.ld;
    for (int j = lane; j < s.need; j += 64) {
      const int64_t at = head + s.first + j;
      row[s.have + j] = c.ring[at < size ? at : at - size];
    }
    for (int j = lane; j < s.back; j += 64) {
      const int64_t at = (int64_t)count + s.first + j;  // behind what was free, as far as the ring has room
      if (at < size) c.ring[head + at < size ? head + at : head + at - size] = row[j];
    }
  }
}

// ------------------------------------------------------------------ rotary positions
//
//   (y_0, y_1) = m (x_0 cos a - x_1 sin a, x_1 cos a + x_0 sin a),  a = 2 pi position turns_i
//
// for pair i of a head.  turns is a 64-bit fraction of a turn, so that position * turns modulo 2^64 is the exact
// remainder of the angle, however far the position, and all its bits count (cos_sin).  A workgroup makes its tokens' cosines and sines once, in LDS, and
// passes over their heads: bound by reading and writing q, k and v once.  8192 tokens, 64 heads over 8 of 128, into the cache:
// 58 us, 5.75 TB/s, and 50 where the inputs are partly in the last cache (a copy of 2 GiB 4.95 TB/s); 16 tokens 3.6 us.
struct RopeCall {
  int T, Hq, Hkv, D, half, interleaved;
  const void *q, *k, *v;
  void *q_out, *k_out, *k_cache, *v_cache;
  size_t q_row, q_head, k_row, k_head, v_row, v_head, qo_row, qo_head, ko_row, ko_head, cache_page, cache_row, cache_head;
  const int32_t *positions, *slots;
  const int64_t *turns;
  float scale, sign;
  int page, slots_end;
  Divider by_page, by_item, by_chunk;
  int tokens;           // of a workgroup
  int per_token;        // items: pieces of 2 PAIRS elements
  int per_head;
};

template <class E>
__device__ __forceinline__ E rounded(float v) {
  if constexpr (sizeof(E) == 2) return to_bf16(v);
  else return v;
}

template <class E, int N>
struct Piece {
  typedef E V __attribute__((ext_vector_type(N)));
  __device__ static __forceinline__ void load(const E *p, E (&x)[N]) {
    if constexpr (N == 1) {
      x[0] = *p;
    } else {
      const V v = *reinterpret_cast<const V *>(p);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = v[i];
    }
  }
  template <bool STREAM>
  __device__ static __forceinline__ void store(E *p, const E (&x)[N]) {
    if constexpr (N == 1) {
      *p = x[0];
    } else {
      V v;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = x[i];
      if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
      else *reinterpret_cast<V *>(p) = v;
    }
  }
};

// An item: a piece of a head of a token, of q, of k or (past both) of v.
template <class E, int PAIRS, bool STREAM>
struct RopeItem {
  int t, h, first, a0, a1;  // first: of its pairs; a0, a1: elements
  bool turned;
  E x[2][PAIRS];
  __device__ __forceinline__ void load(const RopeCall &c, int t0, int e) {
    t = c.by_item(e);
    const int in = e - t * c.per_token;
    h = c.by_chunk(in);
    first = (in - h * c.per_head) * PAIRS;
    const size_t token = (size_t)(t0 + t);
    // pairs of the turned part, then plain ones
    const bool plain = h >= c.Hq + c.Hkv;
    turned = !plain && first < c.half;
    a0 = turned && !c.interleaved ? first : 2 * first;
    a1 = turned && !c.interleaved ? first + c.half : 2 * first + PAIRS;
    const E *from = plain ? static_cast<const E *>(c.v) + token * c.v_row + (size_t)(h - c.Hq - c.Hkv) * c.v_head
                  : h >= c.Hq ? static_cast<const E *>(c.k) + token * c.k_row + (size_t)(h - c.Hq) * c.k_head
                              : static_cast<const E *>(c.q) + token * c.q_row + (size_t)h * c.q_head;
    Piece<E, PAIRS>::load(from + a0, x[0]);
    Piece<E, PAIRS>::load(from + a1, x[1]);
  }
  __device__ __forceinline__ void turn_and_store(const RopeCall &c, int t0, const float2 *angles) {
    const size_t token = (size_t)(t0 + t);
    E y[2][PAIRS];
    if (turned) {
      const float2 *cs = angles + t * c.half + first;
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const float2 w = cs[i];
        if (c.interleaved) {
          E *xs = &x[0][0], *ys = &y[0][0];
          const float u = value(xs[2 * i]), v = value(xs[2 * i + 1]);
          ys[2 * i] = rounded<E>(__builtin_fmaf(u, w.x, -(v * w.y)));
          ys[2 * i + 1] = rounded<E>(__builtin_fmaf(v, w.x, u * w.y));
        } else {
          const float u = value(x[0][i]), v = value(x[1][i]);
          y[0][i] = rounded<E>(__builtin_fmaf(u, w.x, -(v * w.y)));
          y[1][i] = rounded<E>(__builtin_fmaf(v, w.x, u * w.y));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) y[0][i] = x[0][i], y[1][i] = x[1][i];
    }
    auto put = [&](void *rows, size_t at) {
      E *to = static_cast<E *>(rows) + at;
      Piece<E, PAIRS>::template store<STREAM>(to + a0, y[0]);
      Piece<E, PAIRS>::template store<STREAM>(to + a1, y[1]);
    };
    if (h < c.Hq) {
      put(c.q_out, token * c.qo_row + (size_t)h * c.qo_head);
      return;
    }
    const bool key = h < c.Hq + c.Hkv;
    const int head = h - c.Hq - (key ? 0 : c.Hkv);
    if (key && c.k_out != nullptr) put(c.k_out, token * c.ko_row + (size_t)head * c.ko_head);
    // the caches' row, where the token has one
    const int slot = c.slots != nullptr ? c.slots[token] : -1;
    if (slot < 0 || slot >= c.slots_end) return;
    const int index = c.by_page(slot);
    put(key ? c.k_cache : c.v_cache,
        (size_t)index * c.cache_page + (size_t)(slot - index * c.page) * c.cache_row + (size_t)head * c.cache_head);
  }
};

// (cos, sin) of 2 pi phase / 2^64.  Of the nearest whole number of 2^40 that a float holds, then of the rest d, below 2^-24 half
// turns: sin (a + d) = sin a + d cos a, cos (a + d) = cos a - d sin a, d^2 / 2 being below 2^-45.  Rounded to a float as it is,
// the angle would be off by up to 2^-26 of a turn, in small sines by a multiple of their own rounding.
__device__ __forceinline__ float2 cos_sin(int64_t phase) {
  const uint64_t near = (uint64_t)phase + (1ull << 39);   // of all 64 bits: 2^63 is half a turn from either side
  const float whole = (float)((int32_t)(near >> 32) >> 8) * 0x1p-23f;
  const float d = (float)((int64_t)(near & ((1ull << 40) - 1)) - (1ll << 39)) * (float)(3.14159265358979323846 * 0x1p-63);
  float s, c;
  sincospif(whole, &s, &c);
  return float2{__builtin_fmaf(-s, d, c), __builtin_fmaf(c, d, s)};
}

template <class E, int PAIRS, bool STREAM>
__global__ __launch_bounds__(512) void rope_kernel(RopeCall c) {
  extern __shared__ __align__(16) float2 angles[];  // [token][pair]: (cos, sin), scaled
  const int t0 = blockIdx.x * c.tokens, tokens = min(c.tokens, c.T - t0), all = tokens * c.per_token;
  const int stride = blockDim.x * gridDim.y;
  for (int i = threadIdx.x; i < tokens * c.half; i += blockDim.x) {
    const int t = i / c.half, pair = i - t * c.half;
    const int64_t phase = (int64_t)((uint64_t)(int64_t)c.positions[t0 + t] * (uint64_t)c.turns[pair]);
    const float2 w = cos_sin(phase);
    angles[i] = float2{w.x * c.scale, w.y * c.scale * c.sign};
  }
  __syncthreads();
  for (int e = blockIdx.y * blockDim.x + threadIdx.x; e < all; e += stride) {
    RopeItem<E, PAIRS, STREAM> item;
    item.load(c, t0, e);
    item.turn_and_store(c, t0, angles);
  }
}

typedef void (*RopeFn)(RopeCall);

}  // namespace

int kv_tables_launch(const occ_kv_tables_args &a, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  TablesCall c{};
  c.n = a.requests, c.T = a.rows, c.width = a.width, c.pages = a.pages, c.size = a.ring_size, c.page = a.page;
  c.keys = std::min<int64_t>((int64_t)a.width * a.page, OCC_ATTN_MAX_KEYS);
  c.by_page = Divider(a.page);
  c.cached = a.cached, c.fresh = a.fresh, c.free = a.free, c.table = a.table, c.ring = a.ring, c.ld = a.ld_table;
  c.lens = a.lens, c.starts = a.starts, c.slots = a.slots, c.positions = a.positions, c.free_after = a.free_after;
  // a token a thread while that takes no more than two workgroups a CU: each of them scans all requests
  c.each = a.rows <= 2 * kThreads * di->num_cus ? 1 : 4;
  const int grid = std::max({(int)(((int64_t)a.rows + kThreads * c.each - 1) / (kThreads * c.each)), (a.requests + 63) / 64, 1});
  c.requests = (a.requests + grid - 1) / grid;
  hipLaunchKernelGGL(a.requests <= kStaged ? kv_tables_kernel<true> : kv_tables_kernel<false>, dim3(grid), dim3(kThreads), 0, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int rope_launch(const occ_rope_args &a, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  const int Hq = a.q != nullptr ? a.Hq : 0, Hkv = a.k != nullptr ? a.Hkv : 0;
  if (a.rows == 0 || Hq + Hkv == 0) return OCC_OK;
  const bool cache = a.k_cache != nullptr;
  RopeCall c{};
  c.T = a.rows, c.Hq = Hq, c.Hkv = Hkv, c.D = a.D, c.half = a.pairs, c.interleaved = a.interleaved != 0;
  c.q = a.q, c.k = a.k, c.v = a.v, c.q_out = a.q_out, c.k_out = a.k_out, c.k_cache = a.k_cache, c.v_cache = a.v_cache;
  c.q_row = a.q_row, c.q_head = a.q_head, c.k_row = a.k_row, c.k_head = a.k_head, c.v_row = a.v_row, c.v_head = a.v_head;
  c.qo_row = a.qo_row, c.qo_head = a.qo_head, c.ko_row = a.ko_row, c.ko_head = a.ko_head;
  c.cache_page = a.cache_page, c.cache_row = a.cache_row, c.cache_head = a.cache_head;
  c.positions = a.positions, c.slots = cache ? a.slots : nullptr, c.turns = a.turns;
  c.scale = a.scale, c.sign = a.inverse ? -1.f : 1.f;
  c.page = cache ? a.page : 1, c.slots_end = cache ? a.page * a.pages : 0, c.by_page = Divider(c.page);
  // Pieces of as many pairs as 16 bytes hold, where sizes, pitches and addresses are multiples; of one pair otherwise.
  const int elem = a.dtype == OCC_F32 ? 4 : 2;
  auto fits = [&](int pairs) {
    const size_t n = (size_t)pairs, bytes = n * elem;
    size_t all = (size_t)a.pairs | (size_t)a.D / 2;   // both parts are whole pieces
    uintptr_t at = 0;
    if (Hq) all |= a.q_row | a.q_head | a.qo_row | a.qo_head, at |= (uintptr_t)a.q | (uintptr_t)a.q_out;
    if (Hkv) all |= a.k_row | a.k_head, at |= (uintptr_t)a.k;
    if (Hkv && a.k_out) all |= a.ko_row | a.ko_head, at |= (uintptr_t)a.k_out;
    if (cache) all |= a.cache_page | a.cache_row | a.cache_head | a.v_row | a.v_head, at |= (uintptr_t)a.v | (uintptr_t)a.k_cache | (uintptr_t)a.v_cache;
    return a.D % 2 == 0 && all % n == 0 && at % bytes == 0;
  };
  const int pairs = elem == 2 ? (fits(8) ? 8 : fits(4) ? 4 : 1) : (fits(4) ? 4 : 1);
  c.per_head = a.D / 2 / pairs;
  c.per_token = c.per_head * (Hq + Hkv + (cache ? Hkv : 0));
  c.by_item = Divider(c.per_token), c.by_chunk = Divider(c.per_head);
  // More than the L2s hold is stored past them.  8192 tokens, 64 heads over 8 of 128: 77 us with four tokens a workgroup of 256
  // threads and ordinary stores, 62 with one, 50 past the L2s (all with inputs partly in the last cache).
  const RopeGrid grid = rope_grid(a.rows, c.per_token, di->num_cus);
  c.tokens = grid.tokens;
  const bool stream = (int64_t)a.rows * c.per_token * 2 * pairs * elem > (32 << 20);
  RopeFn fn = elem == 2 ? (pairs == 8 ? (stream ? rope_kernel<uint16_t, 8, true> : rope_kernel<uint16_t, 8, false>)
                           : pairs == 4 ? rope_kernel<uint16_t, 4, false> : rope_kernel<uint16_t, 1, false>)
                        : (pairs == 4 ? (stream ? rope_kernel<float, 4, true> : rope_kernel<float, 4, false>) : rope_kernel<float, 1, false>);
  hipLaunchKernelGGL(fn, dim3(grid.x, grid.y), dim3(grid.threads), (size_t)c.tokens * c.half * sizeof(float2), s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace occ
