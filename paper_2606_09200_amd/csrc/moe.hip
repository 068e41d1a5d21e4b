// A whole mixture-of-experts layer for a few tokens (occ_moe).
//
//   l = x Wr^T;  e_1 .. e_k = the k largest of l (ties to the lower index);  p = softmax(l)
//   y = sum_j w_j Wd_j (silu(Wg_j x) * Wu_j x),  w_j = p_j, or p_j / sum of the k
//
// With at most 64 tokens the layer is bound by reading the router and the weights of
// the experts that some token picked, once.  Three launches: the router, whose last
// workgroup picks the experts and lists each one's tokens, and the two products of the
// picked experts, the host not knowing which.  The two products in one launch, the second
// waiting on the device for the first, were slower: tasks then have to come from a
// queue (a workgroup may wait only for work that a running one holds), whose counter
// answers one workgroup every 11 ns (512 of them: 5.8 us), and a kernel's start costs 2.3.
#include "block_util.h"
#include "mx4.h"

#include <algorithm>

namespace occ {
namespace {

constexpr int kMaxTokens = 64, kMaxTopK = 16, kMaxExperts = 512;
constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr uint32_t kNowhere = 0x80000000u;  // a byte offset beyond every descriptor

__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}

template <class V>
__device__ __forceinline__ void put_device(V *p, V v) {  // through the XCD's L2, for readers on other XCDs
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class V>
__device__ __forceinline__ V get_device(const V *p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint32_t add_device(uint32_t *p) {
  return __hip_atomic_fetch_add(p, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The workgroup's device-scope stores have completed before thread 0 goes on.
__device__ __forceinline__ void stores_done() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);
  asm volatile("" ::: "memory");
  __syncthreads();
}

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Largest / smallest of 32-bit words over a wave, in every lane.
template <bool MAX>
__device__ __forceinline__ uint32_t wave_pick(uint32_t v) {
  auto pick = [](uint32_t a, uint32_t b) { return MAX ? max(a, b) : min(a, b); };
  v = pick(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  v = pick(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
  v = pick(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  v = pick(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
  const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = pick(s[0], s[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return pick(t[0], t[1]);
}

// ---------------------------------------------------------------------------
// Router.  A workgroup multiplies 16 experts' rows with all tokens over one of `slices`
// slices of H, its 16 waves 128 columns each in turn; the partial logits go to
// part[slice][token][expert].  The workgroup that arrives last adds the slices in
// order and picks: a wave per token at a time, lane l holding experts l, l + 64, ...
// (PER of them), with the logits of GROUP tokens on their way at once: they come from
// other XCDs' writes through memory, and waiting for each token's in turn made this
// kernel 33 us long for 64 tokens.  Logits order as integers, a NaN below everything
// (its token's weights become NaN with the sum); equal ones go to the lower index.
constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64;

template <int TB, int PER>
__global__ __launch_bounds__(kRouteThreads) void moe_route_kernel(MoeCall c) {
  constexpr int GROUP = PER == 1 ? 4 : PER == 2 ? 2 : 1;
  __shared__ f32x4 partial[kRouteWaves][TB][64];
  __shared__ uint32_t last;
  __shared__ uint32_t picked[kMaxExperts][2];  // the tokens of an expert, a bit each
  __shared__ uint32_t first_of[kMaxExperts];   // its first row of the hidden activations
  __shared__ uint32_t wave_active[kRouteWaves], wave_pairs[kRouteWaves];
  __shared__ float weight_of[kMaxTokens][kMaxTopK];
  __shared__ int id_of[kMaxTokens][kMaxTopK];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int eb = blockIdx.x / c.slices, slice = blockIdx.x % c.slices;
  {
    const int e0 = eb * 16, rows = min(16, c.E - e0);
    const auto rw = rsrc_of(c.router + (size_t)e0 * c.H, (uint32_t)rows * (uint32_t)c.H * 2u);
    const auto rx = rsrc_of(c.x, ((uint32_t)(c.T - 1) * (uint32_t)c.ld_x + (uint32_t)c.H) * 2u);
    f32x4 acc[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t xo[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) xo[b] = b * 16 + l16 < c.T ? (uint32_t)(b * 16 + l16) * (uint32_t)c.ld_x * 2u : kNowhere;
    const int steps = (c.H + 127) / 128;
    for (int s = slice * kRouteWaves + wave; s < steps; s += c.slices * kRouteWaves) {
      u32x4 w[4], x[TB][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t k = (uint32_t)(s * 128 + i * 32 + g * 8);
        const bool in = k < (uint32_t)c.H;
        w[i] = load16(rw, in ? ((uint32_t)l16 * (uint32_t)c.H + k) * 2u : kNowhere);
#pragma unroll
        for (int b = 0; b < TB; ++b) x[b][i] = load16(rx, in ? xo[b] + k * 2u : kNowhere);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[b] = mfma_bf16(w[i], x[b][i], acc[b]);
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) partial[wave][b][lane] = acc[b];
    __syncthreads();
    if (wave < TB) {
      f32x4 v = partial[0][wave][lane];
#pragma unroll
      for (int w = 1; w < kRouteWaves; ++w) v = v + partial[w][wave][lane];
      const int t = wave * 16 + l16;
      if (t < c.T) {
        float *p = c.part + ((size_t)slice * c.T + t) * c.E;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (e0 + g * 4 + i < c.E) put_device(p + e0 + g * 4 + i, v[i]);
      }
    }
  }
  stores_done();
  if (threadIdx.x == 0) last = add_device(&c.count->arrived) + 1 == gridDim.x;
  __syncthreads();
  if (!last) return;

  if (threadIdx.x == 0) put_device(&c.count->arrived, 0u);  // for the next call
  for (int i = threadIdx.x; i < c.row_blocks; i += kRouteThreads) c.joined[i] = 0;
  for (int i = threadIdx.x; i < c.E; i += kRouteThreads) picked[i][0] = picked[i][1] = 0u;
  __syncthreads();
  for (int t0 = wave * GROUP; t0 < c.T; t0 += kRouteWaves * GROUP) {
    float logit[GROUP][PER];
#pragma unroll
    for (int q = 0; q < GROUP; ++q)
#pragma unroll
      for (int j = 0; j < PER; ++j) logit[q][j] = 0.f;
#pragma unroll 2
    for (int s = 0; s < c.slices; ++s) {
      float v[GROUP][PER];
#pragma unroll
      for (int q = 0; q < GROUP; ++q)
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const int t = min(t0 + q, c.T - 1), e = min(j * 64 + lane, c.E - 1);
          v[q][j] = get_device(c.part + ((size_t)s * c.T + t) * c.E + e);
        }
#pragma unroll
      for (int q = 0; q < GROUP; ++q)
#pragma unroll
        for (int j = 0; j < PER; ++j) logit[q][j] = logit[q][j] + v[q][j];
    }
#pragma unroll
    for (int q = 0; q < GROUP; ++q) {
      const int t = t0 + q;
      if (t >= c.T) break;
      if (c.mask != nullptr && c.mask[t] == 0) {
        if (lane < c.k) {
          if (c.ids != nullptr) c.ids[t * c.k + lane] = -1;
          if (c.weights != nullptr) c.weights[t * c.k + lane] = 0.f;
          id_of[t][lane] = -1;
        }
        continue;
      }
      float l[PER];
      uint32_t key[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        l[j] = logit[q][j];
        // ascending integers, 1 and above; what is taken or missing is 0
        const uint32_t u = __builtin_bit_cast(uint32_t, l[j]);
        key[j] = j * 64 + lane >= c.E ? 0u : l[j] != l[j] ? 1u : (u >> 31 ? ~u : u | 0x80000000u);
      }
      float top = 0.f, mine = 0.f;  // mine: lane j < k holds pick j's logit, then its weight
      int my_id = 0;
      for (int j = 0; j < c.k; ++j) {
        uint32_t best = 0u;
        int at = 0;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
          if (key[i] >= best) best = key[i], at = i;  // the lowest index among this lane's equals
        const uint32_t win = wave_pick<true>(best);
        const uint32_t e = wave_pick<false>(best == win ? (uint32_t)(at * 64 + lane) : 0xFFFFFFFFu);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if ((uint32_t)(i * 64 + lane) == e) v = l[i], key[i] = 0u;
        v = as_float((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, v), (int)(e & 63u)));
        if (j == 0) top = v;
        if (lane == j) mine = v, my_id = (int)e;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i * 64 + lane < c.E) sum = sum + expf(l[i] - top);
      sum = wave_sum(sum);
      mine = lane < c.k ? expf(mine - top) : 0.f;
      const float kept = wave_sum(mine);
      // a NaN among the logits is in `sum`, whichever experts were picked
      mine = c.renorm ? (sum == sum ? mine / kept : sum) : mine / sum;
      if (lane < c.k) {
        if (c.ids != nullptr) c.ids[t * c.k + lane] = my_id;
        if (c.weights != nullptr) c.weights[t * c.k + lane] = mine;
        id_of[t][lane] = my_id;
        weight_of[t][lane] = mine;
        atomicOr(&picked[my_id][t >> 5], 1u << (t & 31));
      }
    }
  }
  __syncthreads();
  // active experts in index order, with the first of their rows of the hidden activations
  const int e = threadIdx.x;
  const uint32_t m0 = e < c.E ? picked[e][0] : 0u, m1 = e < c.E ? picked[e][1] : 0u;
  const int n = __popc(m0) + __popc(m1);
  const uint64_t act = __ballot(n > 0);
  int before = n;  // pairs of lower lanes
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(before, d);
    if (lane >= d) before += o;
  }
  if (lane == 63) wave_pairs[wave] = before;
  if (lane == 0) wave_active[wave] = __popcll(act);
  before -= n;
  __syncthreads();
  int slot = __popcll(act & ((1ull << lane) - 1)), total = 0;
#pragma unroll
  for (int w = 0; w < kRouteWaves; ++w) {
    if (w < wave) slot += wave_active[w], before += wave_pairs[w];
    total += wave_active[w];
  }
  if (threadIdx.x == 0) c.count->active = total;
  if (n > 0) {
    c.plan[slot] = MoeExpert{(uint32_t)e, (uint32_t)before, (uint32_t)n, 0u};
    first_of[e] = (uint32_t)before;
  }
  __syncthreads();
  // an expert's rows are its tokens in order
  for (int i = threadIdx.x; i < c.T * c.k; i += kRouteThreads) {
    const int t = i / c.k, id = id_of[t][i % c.k];
    if (id < 0) continue;
    const uint64_t m = (uint64_t)picked[id][1] << 32 | picked[id][0];
    c.rows[first_of[id] + __popcll(m & ((1ull << t) - 1))] = MoeRow{t, weight_of[t][i % c.k]};
  }
}

// ---------------------------------------------------------------------------
// A 16-row block of an expert's matrix, read in steps of 128 columns: four MFMA
// operands of 32 columns.  bf16: operand i is columns 32 i + 8 g .. + 7 of lane (row, g).
// MX4: a lane's 16 bytes are the block of columns 32 g .. + 31, operand i its columns
// 8 i .. + 7, converted to bf16 exactly (E2M1 has two bits of precision) with the block's
// scale; the other factor is read in the same order.
template <bool MX>
struct Rows16;
template <>
struct Rows16<false> {
  struct Step {
    u32x4 w[4];
  };
  __amdgpu_buffer_rsrc_t r;
  uint32_t at, cols;
  static __device__ __forceinline__ uint32_t column(int i, int g) { return 32 * i + 8 * g; }
  __device__ __forceinline__ Rows16(const MoeMatrix &m, int e, int row0, int rows, int cols_, int lane) : cols(cols_) {
    r = rsrc_of(static_cast<const uint8_t *>(m.w) + (size_t)e * m.stride + (size_t)row0 * cols * 2,
                (uint32_t)min(16, rows - row0) * cols * 2u);
    at = (uint32_t)(lane & 15) * cols * 2u;
  }
  __device__ __forceinline__ void load(Step &s, int step, int lane, bool in) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t k = (uint32_t)step * 128u + column(i, lane >> 4);
      s.w[i] = load16(r, in && k < cols ? at + k * 2u : kNowhere);
    }
  }
  static __device__ __forceinline__ u32x4 operand(const Step &s, int i) { return s.w[i]; }
};
template <>
struct Rows16<true> {
  struct Step {
    u32x4 w;
    uint32_t s;
  };
  __amdgpu_buffer_rsrc_t r, rs;
  uint32_t at;
  static __device__ __forceinline__ uint32_t column(int i, int g) { return 32 * g + 8 * i; }
  __device__ __forceinline__ Rows16(const MoeMatrix &m, int e, int row0, int rows, int cols, int lane) {
    const uint32_t P = (uint32_t)(OCC_MX4_KP(cols) / 2);
    r = rsrc_of(static_cast<const uint8_t *>(m.w) + (size_t)e * m.stride + (size_t)row0 * P, (uint32_t)min(16, rows - row0) * P);
    rs = rsrc_of(m.scales + (size_t)e * m.scale_stride + (size_t)(row0 >> 4) * P, P);
    at = (uint32_t)(lane & 15) * P + (uint32_t)(lane >> 4) * 16u;
  }
  __device__ __forceinline__ void load(Step &s, int step, int lane, bool in) const {
    s.w = load16(r, in ? at + (uint32_t)step * 64u : kNowhere);
    s.s = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)(in ? (uint32_t)(step >> 2) * 256u + lane * 4u + (step & 3) : kNowhere), 0, 0);
  }
  static __device__ __forceinline__ u32x4 operand(const Step &s, int i) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const float sc = mx4_scale_value(s.s);
    const uint32_t w = s.w[i];
    u32x4 o;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3);
    o[0] = __builtin_bit_cast(uint32_t, a);
    o[1] = __builtin_bit_cast(uint32_t, b);
    o[2] = __builtin_bit_cast(uint32_t, c);
    o[3] = __builtin_bit_cast(uint32_t, d);
    // the conversion takes the scale's exponent alone; a NaN scale (a block that held one) stays NaN
    if (s.s == 255u) o = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
    return o;
  }
};

// What the router left, read through the scalar cache: the kernels below only read it.
__device__ __forceinline__ MoeExpert expert_at(const MoeCall &c, uint32_t i) {
  typedef const __attribute__((address_space(4))) MoeExpert *Constant;
  const Constant p = (Constant)(uintptr_t)c.plan;
  MoeExpert e;
  e.id = __builtin_amdgcn_readfirstlane(p[i].id);
  e.first = __builtin_amdgcn_readfirstlane(p[i].first);
  e.n = __builtin_amdgcn_readfirstlane(p[i].n);
  return e;
}

// The other factor's operands of steps b U .. b U + U - 1: rows at byte offset `from`.
template <class Rows, int U>
__device__ __forceinline__ void factor(u32x4 (&x)[U][4], __amdgpu_buffer_rsrc_t r, uint32_t from, int b, int cols, int g) {
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t k = (uint32_t)(b * U + u) * 128u + Rows::column(i, g);
      x[u][i] = load16(r, k < (uint32_t)cols ? from + k * 2u : kNowhere);
    }
}

template <bool MX>
constexpr int kBatch = MX ? 2 : 1;  // 128-column steps of a batch

// ---------------------------------------------------------------------------
// silu(Wg x) * (Wu x).  A task is 16 rows of Wg and of Wu of one expert with that expert's
// tokens (16 to an MFMA); the 8 waves split H, the sums meet in LDS in wave order, and
// the result is rounded to bf16, the next product's operand.
//
// What bounds it is the stream of weights, so it must not stop: a wave has the next
// batch's weights in flight while it multiplies (loads return in order: the other
// factor's and the next task's rows are asked for before them), also across the end of a
// task, and two workgroups share a CU.
template <bool MX, int TB>
__global__ __launch_bounds__(kThreads, TB > 2 ? 2 : 4) void moe_up_kernel(MoeCall c) {
  constexpr int U = kBatch<MX>;
  typedef Rows16<MX> Rows;
  __shared__ f32x4 sums[TB > 2 ? 1 : 2][kWaves][TB][2][64];  // used in turn where two fit beside another workgroup's
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t blocks = (uint32_t)(c.I + 15) / 16;
  const uint32_t tasks = __builtin_amdgcn_readfirstlane(c.count->active) * blocks;
  if (blockIdx.x >= tasks) return;
  const auto rx = rsrc_of(c.x, ((uint32_t)(c.T - 1) * (uint32_t)c.ld_x + (uint32_t)c.H) * 2u);
  const int batches = (c.H + 128 * U - 1) / (128 * U);
  const int b0 = wave * batches / kWaves, b1 = (wave + 1) * batches / kWaves;
  typename Rows::Step wg[U], wu[U];
  auto load = [&](const MoeExpert &e, uint32_t task, int b) {
    const int row0 = (int)(task % blocks) * 16;
    const Rows rg(c.gate, (int)e.id, row0, c.I, c.H, lane), ru(c.up, (int)e.id, row0, c.I, c.H, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      rg.load(wg[u], b * U + u, lane, (b * U + u) * 128 < c.H);
      ru.load(wu[u], b * U + u, lane, (b * U + u) * 128 < c.H);
    }
  };
  int token[TB];  // of this lane's column in each 16, -1 past the last
  auto tokens_of = [&](const MoeExpert &e) {
#pragma unroll
    for (int at = 0; at < TB; ++at) token[at] = at * 16 + l16 < (int)e.n ? c.rows[e.first + at * 16 + l16].token : -1;
  };
  MoeExpert ex = expert_at(c, blockIdx.x / blocks);
  tokens_of(ex);
  if (b0 < b1) load(ex, blockIdx.x, b0);
  int turn = 0;
  for (uint32_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const uint32_t nxt = task + gridDim.x;
    const MoeExpert en = nxt < tasks ? expert_at(c, nxt / blocks) : ex;
    const int n = (int)ex.n, nb = (n + 15) / 16;
    f32x4 ag[TB], au[TB];
    uint32_t xo[TB];
#pragma unroll
    for (int at = 0; at < TB; ++at) {
      ag[at] = au[at] = f32x4{0.f, 0.f, 0.f, 0.f};
      xo[at] = token[at] >= 0 ? (uint32_t)token[at] * (uint32_t)c.ld_x * 2u : kNowhere;
    }
    for (int b = b0; b < b1; ++b) {
      u32x4 x[U][4];
      factor<Rows, U>(x, rx, xo[0], b, c.H, g);
      typename Rows::Step fg[U], fu[U];
#pragma unroll
      for (int u = 0; u < U; ++u) fg[u] = wg[u], fu[u] = wu[u];
      if (b + 1 == b1 && nxt < tasks) tokens_of(en);
      __builtin_amdgcn_sched_barrier(0);
      if (b + 1 < b1) load(ex, task, b + 1);
      else if (nxt < tasks) load(en, nxt, b0);
      __builtin_amdgcn_sched_barrier(0);
      auto multiply = [&](int at) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ag[at] = mfma_bf16(Rows::operand(fg[u], i), x[u][i], ag[at]);
            au[at] = mfma_bf16(Rows::operand(fu[u], i), x[u][i], au[at]);
          }
      };
      multiply(0);
#pragma unroll
      for (int at = 1; at < TB; ++at)
        if (at < nb) {
          factor<Rows, U>(x, rx, xo[at], b, c.H, g);
          multiply(at);
        }
    }
    if (b0 == b1 && nxt < tasks) tokens_of(en);
    auto &part = sums[turn];
#pragma unroll
    for (int at = 0; at < TB; ++at)
      if (at < nb) {
        part[wave][at][0][lane] = ag[at];
        part[wave][at][1][lane] = au[at];
      }
    __syncthreads();
    if (wave < nb) {
      f32x4 gs = part[0][wave][0][lane], us = part[0][wave][1][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) {
        gs = gs + part[w][wave][0][lane];
        us = us + part[w][wave][1][lane];
      }
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = gs[i] / (1.f + expf(-gs[i])) * us[i];
      const int row = (int)(task % blocks) * 16 + g * 4;  // I is a multiple of 8: all four exist or none
      if (wave * 16 + l16 < n && row < c.I)
        *reinterpret_cast<uint64_t *>(c.hidden + (size_t)(ex.first + wave * 16 + l16) * c.I + row) =
            (uint64_t)pack_bf16(v[2], v[3]) << 32 | pack_bf16(v[0], v[1]);
    }
    if constexpr (TB > 2) __syncthreads();
    else turn ^= 1;
    ex = en;
  }
}

// ---------------------------------------------------------------------------
// y = sum_j w_j Wd_j h_j.  A task is 16 rows of Wd for the experts of one of `segments` parts
// of the list; the waves split those experts' columns end to end, each adding its
// experts' weighted sums to its own rows of y in LDS, one per token (a token that did not
// pick an expert gets nothing from it, whatever its weights hold).  With several segments
// the last one to finish a row block adds them in order: no sum depends on timing.
// The weights' stream is kept up as above.
template <bool MX, int TB>
__global__ __launch_bounds__(kThreads, TB > 2 ? 2 : 4) void moe_down_kernel(MoeCall c) {
  constexpr int U = 2;  // 128-column steps of a batch
  typedef Rows16<MX> Rows;
  extern __shared__ __align__(16) unsigned char smem[];  // two areas [wave][token][16 rows], used in turn
  __shared__ uint32_t last;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int active = (int)__builtin_amdgcn_readfirstlane(c.count->active);
  const int segments = max(1, min(active, c.max_segments));
  const int tasks = c.row_blocks * segments;
  if ((int)blockIdx.x >= tasks) return;
  const auto rh = rsrc_of(c.hidden, (uint32_t)(c.T * c.k) * (uint32_t)c.I * 2u);
  const int batches = (c.I + 128 * U - 1) / (128 * U);  // of one expert
  const int area_floats = kWaves * c.T * 16;
  typename Rows::Step wd[U];
  struct Part {  // of a task: its rows, its first expert, and this wave's batches of all its experts, end to end
    int row0, a0, b0, b1;
  };
  auto part_of = [&](int task) {
    const int seg = task % segments;
    Part p;
    p.row0 = task / segments * 16;
    p.a0 = seg * active / segments;
    const int all = ((seg + 1) * active / segments - p.a0) * batches;
    p.b0 = wave * all / kWaves;
    p.b1 = (wave + 1) * all / kWaves;
    return p;
  };
  auto load = [&](const Part &p, int b) {
    const Rows rd(c.down, (int)expert_at(c, p.a0 + b / batches).id, p.row0, c.H, c.I, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = b % batches * U + u;
      rd.load(wd[u], s, lane, s * 128 < c.I);
    }
  };
  Part p = part_of(blockIdx.x);
  if (p.b0 < p.b1) load(p, p.b0);
  int turn = 0;
  for (int task = blockIdx.x; task < tasks; task += gridDim.x, turn ^= 1) {
    Part q{0, 0, 0, 0};
    if (task + (int)gridDim.x < tasks) q = part_of(task + gridDim.x);
    float *area = reinterpret_cast<float *>(smem) + turn * area_floats, *mine = area + wave * c.T * 16;
    for (int i = lane; i < c.T * 4; i += 64) reinterpret_cast<f32x4 *>(mine)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int b = p.b0; b < p.b1;) {
      const MoeExpert ex = expert_at(c, p.a0 + b / batches);
      const int n = (int)ex.n, nb = (n + 15) / 16;
      const int end = min(p.b1, (b / batches + 1) * batches);
      f32x4 acc[TB];
      uint32_t ho[TB];
#pragma unroll
      for (int at = 0; at < TB; ++at) {
        acc[at] = f32x4{0.f, 0.f, 0.f, 0.f};
        ho[at] = at * 16 + l16 < n ? (ex.first + at * 16 + l16) * (uint32_t)c.I * 2u : kNowhere;
      }
      MoeRow row[TB];
      for (; b < end; ++b) {
        u32x4 x[U][4];
        factor<Rows, U>(x, rh, ho[0], b % batches, c.I, g);
        typename Rows::Step fd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) fd[u] = wd[u];
        if (b + 1 == end) {
#pragma unroll
          for (int at = 0; at < TB; ++at)
            if (at * 16 + l16 < n) row[at] = c.rows[ex.first + at * 16 + l16];
        }
        __builtin_amdgcn_sched_barrier(0);
        if (b + 1 < p.b1) load(p, b + 1);
        else if (q.b0 < q.b1) load(q, q.b0);
        __builtin_amdgcn_sched_barrier(0);
        auto multiply = [&](int at) {
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[at] = mfma_bf16(Rows::operand(fd[u], i), x[u][i], acc[at]);
        };
        multiply(0);
#pragma unroll
        for (int at = 1; at < TB; ++at)
          if (at < nb) {
            factor<Rows, U>(x, rh, ho[at], b % batches, c.I, g);
            multiply(at);
          }
      }
      // this wave's part of the expert is whole: into its tokens' rows
#pragma unroll
      for (int at = 0; at < TB; ++at)
        if (at * 16 + l16 < n) {
          f32x4 *y = reinterpret_cast<f32x4 *>(mine + row[at].token * 16 + g * 4);
          f32x4 v = *y;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(row[at].weight, acc[at][i], v[i]);
          *y = v;
        }
    }
    if (p.b0 == p.b1 && q.b0 < q.b1) load(q, q.b0);
    __syncthreads();
    const int rb = p.row0 / 16, seg = task % segments;
    const int tok = threadIdx.x >> 2, row = p.row0 + (threadIdx.x & 3) * 4;  // H is a multiple of 8
    const bool has = tok < c.T && row < c.H;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (has) {
      const f32x4 *in = reinterpret_cast<const f32x4 *>(area) + threadIdx.x;
      v = in[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v = v + in[w * c.T * 4];
    }
    bool store = has;
    if (segments > 1) {
      const size_t at = (size_t)tok * c.H + row, whole = (size_t)c.T * c.H;
      if (has) {
#pragma unroll
        for (int i = 0; i < 4; ++i) put_device(c.sums + seg * whole + at + i, v[i]);
      }
      stores_done();
      if (threadIdx.x == 0) last = add_device(c.joined + rb) + 1 == (uint32_t)segments;
      __syncthreads();
      store = has && last;
      if (store) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = get_device(c.sums + at + i);
        for (int s = 1; s < segments; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = v[i] + get_device(c.sums + s * whole + at + i);
      }
    }
    if (store) {
      typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
      u32x2_e2 o;
      o[0] = pack_bf16(v[0], v[1]);
      o[1] = pack_bf16(v[2], v[3]);
      *reinterpret_cast<u32x2_e2 *>(c.y + (size_t)tok * c.ld_y + row) = o;
    }
    p = q;
  }
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// The workspace's parts; the counters come first.
struct MoeLayout {
  size_t plan, rows, joined, part, hidden, sums, end;
  int slices, segments, row_blocks;
};
MoeLayout layout_of(int T, int H, int I, int E, int k) {
  MoeLayout l{};
  l.slices = std::max(1, std::min(16, (H + 128 * kRouteWaves - 1) / (128 * kRouteWaves)));  // one step a wave
  l.row_blocks = (H + 15) / 16;
  // parts of the second kind's tasks: two tasks a workgroup or more, so that the last ones to end
  // are short, with at most E experts to share
  l.segments = std::max(1, std::min(std::min(E, T * k), (1024 + l.row_blocks - 1) / l.row_blocks));
  size_t at = up16(sizeof(MoeCounters));
  l.plan = at, at += up16((size_t)E * sizeof(MoeExpert));
  l.rows = at, at += up16((size_t)T * k * sizeof(MoeRow));
  l.joined = at, at += up16((size_t)l.row_blocks * 4);
  l.part = at, at += up16((size_t)l.slices * T * E * 4);
  l.hidden = at, at += up16((size_t)T * k * I * 2);
  l.sums = at, at += up16(l.segments > 1 ? (size_t)l.segments * T * H * 4 : 0);
  l.end = at;
  return l;
}

typedef void (*MoeFn)(MoeCall);
template <int PER>
MoeFn route_fn(int tb) {
  return tb == 1 ? moe_route_kernel<1, PER> : tb == 2 ? moe_route_kernel<2, PER> : moe_route_kernel<4, PER>;
}
template <bool MX>
MoeFn up_fn(int tb) {
  return tb == 1 ? moe_up_kernel<MX, 1> : tb == 2 ? moe_up_kernel<MX, 2> : moe_up_kernel<MX, 4>;
}
template <bool MX>
MoeFn down_fn(int tb) {
  return tb == 1 ? moe_down_kernel<MX, 1> : tb == 2 ? moe_down_kernel<MX, 2> : moe_down_kernel<MX, 4>;
}

}  // namespace

size_t moe_workspace(int T, int H, int I, int E, int k) { return layout_of(T, H, I, E, k).end; }

int moe_launch(const occ_moe_args &a, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (a.tokens == 0) return OCC_OK;
  const MoeLayout l = layout_of(a.tokens, a.H, a.I, a.experts, a.top_k);
  unsigned char *ws = static_cast<unsigned char *>(a.workspace);
  MoeCall c{};
  c.T = a.tokens, c.H = a.H, c.I = a.I, c.E = a.experts, c.k = a.top_k, c.renorm = a.renorm != 0;
  c.slices = l.slices, c.row_blocks = l.row_blocks, c.max_segments = l.segments;
  c.x = static_cast<const uint16_t *>(a.x), c.ld_x = (int)a.ld_x;
  c.router = static_cast<const uint16_t *>(a.router);
  const bool mx = a.weight_type == OCC_MX4;
  auto matrix = [&](const void *w, const void *scales, size_t stride, int rows, int cols) {
    const size_t packed = mx ? OCC_MX4_CODE_BYTES(rows, cols) : (size_t)rows * cols * 2;
    return MoeMatrix{w, static_cast<const uint8_t *>(scales), mx || stride == 0 ? packed : stride * 2,
                     OCC_MX4_SCALE_BYTES(rows, cols)};
  };
  c.gate = matrix(a.w_gate, a.s_gate, a.stride_gate, a.I, a.H);
  c.up = matrix(a.w_up, a.s_up, a.stride_up, a.I, a.H);
  c.down = matrix(a.w_down, a.s_down, a.stride_down, a.H, a.I);
  c.mask = static_cast<const uint8_t *>(a.mask);
  c.y = static_cast<uint16_t *>(a.y), c.ld_y = a.ld_y, c.ids = a.ids, c.weights = a.weights;
  c.count = reinterpret_cast<MoeCounters *>(ws);
  c.plan = reinterpret_cast<MoeExpert *>(ws + l.plan);
  c.rows = reinterpret_cast<MoeRow *>(ws + l.rows);
  c.joined = reinterpret_cast<uint32_t *>(ws + l.joined);
  c.part = reinterpret_cast<float *>(ws + l.part);
  c.hidden = reinterpret_cast<uint16_t *>(ws + l.hidden);
  c.sums = reinterpret_cast<float *>(ws + l.sums);
  const int tb = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
  const MoeFn route = a.experts <= 64 ? route_fn<1>(tb) : a.experts <= 128 ? route_fn<2>(tb) : route_fn<8>(tb);
  hipLaunchKernelGGL(route, dim3((a.experts + 15) / 16 * l.slices), dim3(kRouteThreads), 0, s, c);
  if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  const unsigned grid = (unsigned)di->num_cus * 2;
  hipLaunchKernelGGL(mx ? up_fn<true>(tb) : up_fn<false>(tb), dim3(grid), dim3(kThreads), 0, s, c);
  if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  hipLaunchKernelGGL(mx ? down_fn<true>(tb) : down_fn<false>(tb), dim3(grid), dim3(kThreads), 2 * kWaves * a.tokens * 64, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int validate_moe_sizes(int T, int H, int I, int E, int k) {
  if (T < 0 || T > kMaxTokens || E < 1 || E > kMaxExperts || k < 1 || k > kMaxTopK || k > E) return OCC_EINVAL;
  if (H < 8 || H > 65536 || H % 8 != 0 || I < 8 || I > 65536 || I % 8 != 0) return OCC_EINVAL;
  return OCC_OK;
}

}  // namespace occ
