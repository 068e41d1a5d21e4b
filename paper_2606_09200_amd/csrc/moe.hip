// A whole mixture-of-experts layer for a few tokens (occ_moe).
//
//   l = x Wr^T;  e_1 .. e_k = the k largest of l (ties to the lower index);  p = softmax(l)
//   y = sum_j w_j Wd_j (silu(Wg_j x) * Wu_j x),  w_j = p_j, or p_j / sum of the k
//
// With at most 64 tokens the layer is bound by reading the router and the weights of
// the experts that some token picked, once.  Two kernels: the router, whose last
// workgroup picks the experts and lists each one's tokens, and the experts, whose
// workgroups take tasks from a queue: first all (expert, 16 rows of Wg and Wu), then
// all (16 rows of Wd, experts).
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
// slices of H, its 8 waves 128 columns each in turn; the partial logits go to
// part[slice][token][expert].  The workgroup that arrives last adds the slices in
// order and picks: a wave per token at a time, lane l holding experts l, l + 64, ...
// Logits order as integers, a NaN below everything (its token's weights become NaN
// with the sum); equal ones go to the lower index.
template <int TB>
__global__ __launch_bounds__(kThreads) void moe_route_kernel(MoeCall c) {
  __shared__ f32x4 partial[kWaves][TB][64];
  __shared__ uint32_t last;
  __shared__ uint32_t picked[kMaxExperts][2];  // the tokens of an expert, a bit each
  __shared__ uint32_t wave_active[kWaves], wave_pairs[kWaves];
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
    for (int s = slice * kWaves + wave; s < steps; s += c.slices * kWaves) {
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
      for (int w = 1; w < kWaves; ++w) v = v + partial[w][wave][lane];
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

  if (threadIdx.x == 0) {  // for the next call's router and this call's experts
    put_device(&c.count->arrived, 0u);
    c.count->ticket = 0;
    c.count->up_done = 0;
  }
  for (int i = threadIdx.x; i < c.row_blocks; i += kThreads) c.joined[i] = 0;
  for (int i = threadIdx.x; i < c.E; i += kThreads) picked[i][0] = picked[i][1] = 0u;
  __syncthreads();
  constexpr int PER = kMaxExperts / 64;
  for (int t = wave; t < c.T; t += kWaves) {
    if (c.mask != nullptr && c.mask[t] == 0) {
      if (lane < c.k) {
        if (c.ids != nullptr) c.ids[t * c.k + lane] = -1;
        if (c.weights != nullptr) c.weights[t * c.k + lane] = 0.f;
      }
      continue;
    }
    float l[PER];
    uint32_t key[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int e = j * 64 + lane;
      l[j] = 0.f;
      key[j] = 0u;
      if (j * 64 < c.E && e < c.E) {
        const float *p = c.part + (size_t)t * c.E + e;
        for (int s = 0; s < c.slices; ++s) l[j] = l[j] + get_device(p + (size_t)s * c.T * c.E);
        // ascending integers, 1 and above; what is taken or missing is 0
        const uint32_t u = __builtin_bit_cast(uint32_t, l[j]);
        key[j] = l[j] != l[j] ? 1u : (u >> 31 ? ~u : u | 0x80000000u);
      }
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
      c.gate_of[(size_t)my_id * kMaxTokens + t] = mine;
      atomicOr(&picked[my_id][t >> 5], 1u << (t & 31));
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
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) slot += wave_active[w], before += wave_pairs[w];
    total += wave_active[w];
  }
  if (threadIdx.x == 0) c.count->active = total;
  if (n > 0) {
    c.plan[slot] = MoeExpert{(uint32_t)e, (uint32_t)before, {m0, m1}};
    int r = before;
    for (uint64_t m = (uint64_t)m1 << 32 | m0; m != 0; m &= m - 1) c.token_of[r++] = __builtin_ctzll(m);
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

// Experts.  Tasks are taken in order from a queue, so a task is held by a workgroup that
// runs, and workgroups that wait for all tasks of the first kind hold none of them:
// the wait ends whatever else occupies the GPU.
//
// First kind: 16 rows of Wg and of Wu of one expert with that expert's tokens (16 to an
// MFMA); the 8 waves split H, the sums meet in LDS, silu(g) u is rounded to bf16, the
// next product's operand, and stored at device scope.  Second kind: 16 rows of Wd for
// the experts of one of `segments` parts of the list; the waves split I, an MFMA's
// columns are the tokens themselves, and a token's weighted sum over its experts
// stays in the lane's registers.  With several segments the last one to finish a row
// block adds them in order.  No sum depends on timing.
template <bool MX, int TB>
__global__ __launch_bounds__(kThreads) void moe_experts_kernel(MoeCall c) {
  constexpr int U = MX ? 4 : 2;  // 128-column steps in flight
  typedef Rows16<MX> Rows;
  __shared__ f32x4 partial[kWaves][2 * TB][64];
  __shared__ uint32_t ticket, last;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int active = __builtin_amdgcn_readfirstlane((int)c.count->active);
  const int up_blocks = (c.I + 15) / 16;
  const uint32_t ups = (uint32_t)active * up_blocks;
  // enough second-kind tasks for every workgroup, but no more parts than experts
  const int segments = max(1, min(min(active, c.max_segments), ((int)gridDim.x + c.row_blocks - 1) / c.row_blocks));
  const uint32_t tasks = ups + (uint32_t)(c.row_blocks * segments);
  const auto rx = rsrc_of(c.x, ((uint32_t)(c.T - 1) * (uint32_t)c.ld_x + (uint32_t)c.H) * 2u);
  const auto rh = rsrc_of(c.hidden, (uint32_t)(c.T * c.k) * (uint32_t)c.I * 2u);
  bool waited = false;

  if (threadIdx.x == 0) ticket = add_device(&c.count->ticket);
  __syncthreads();
  for (uint32_t task = ticket; task < tasks;) {
    uint32_t next = 0;
    if (threadIdx.x == 0) next = add_device(&c.count->ticket);  // arrives while this task runs
    if (task < ups) {
      const MoeExpert ex = c.plan[task / up_blocks];
      const int row0 = (int)(task % up_blocks) * 16;
      const int n = __popc(ex.tokens[0]) + __popc(ex.tokens[1]), nb = (n + 15) / 16;
      const Rows wg(c.gate, ex.id, row0, c.I, c.H, lane), wu(c.up, ex.id, row0, c.I, c.H, lane);
      uint32_t xo[TB];
#pragma unroll
      for (int b = 0; b < TB; ++b)
        xo[b] = b * 16 + l16 < n ? (uint32_t)c.token_of[ex.first + b * 16 + l16] * (uint32_t)c.ld_x * 2u : kNowhere;
      f32x4 ag[TB], au[TB];
#pragma unroll
      for (int b = 0; b < TB; ++b) ag[b] = au[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int steps = (c.H + 127) / 128;
      for (int s = wave * U; s < steps; s += kWaves * U) {
        typename Rows::Step fg[U], fu[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          wg.load(fg[u], s + u, lane, s + u < steps);
          wu.load(fu[u], s + u, lane, s + u < steps);
        }
#pragma unroll
        for (int b = 0; b < TB; ++b)
          if (b < nb) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t k = (uint32_t)(s + u) * 128u + Rows::column(i, g);
                const u32x4 x = load16(rx, k < (uint32_t)c.H ? xo[b] + k * 2u : kNowhere);
                ag[b] = mfma_bf16(Rows::operand(fg[u], i), x, ag[b]);
                au[b] = mfma_bf16(Rows::operand(fu[u], i), x, au[b]);
              }
          }
      }
#pragma unroll
      for (int b = 0; b < TB; ++b)
        if (b < nb) {
          partial[wave][2 * b][lane] = ag[b];
          partial[wave][2 * b + 1][lane] = au[b];
        }
      __syncthreads();
      if (wave < nb) {
        f32x4 gs = partial[0][2 * wave][lane], us = partial[0][2 * wave + 1][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
          gs = gs + partial[w][2 * wave][lane];
          us = us + partial[w][2 * wave + 1][lane];
        }
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gs[i] / (1.f + expf(-gs[i])) * us[i];
        const int row = row0 + g * 4;  // I is a multiple of 8: all four exist or none
        if (wave * 16 + l16 < n && row < c.I)
          put_device(reinterpret_cast<uint64_t *>(c.hidden + (size_t)(ex.first + wave * 16 + l16) * c.I + row),
                     (uint64_t)pack_bf16(v[2], v[3]) << 32 | pack_bf16(v[0], v[1]));
      }
      stores_done();
      if (threadIdx.x == 0) add_device(&c.count->up_done);
    } else {
      if (!waited) {
        if (threadIdx.x == 0)
          while (get_device(&c.count->up_done) < ups) __builtin_amdgcn_s_sleep(2);
        __syncthreads();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");  // once a workgroup
        waited = true;
      }
      const int rb = (int)(task - ups) / segments, seg = (int)(task - ups) % segments;
      const int row0 = rb * 16;
      const int a0 = seg * active / segments, a1 = (seg + 1) * active / segments;
      f32x4 y[TB];
#pragma unroll
      for (int b = 0; b < TB; ++b) y[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int steps = (c.I + 127) / 128;
      for (int a = a0; a < a1; ++a) {
        const MoeExpert ex = c.plan[a];
        const uint64_t tokens = (uint64_t)ex.tokens[1] << 32 | ex.tokens[0];
        const Rows wd(c.down, ex.id, row0, c.H, c.I, lane);
        uint32_t ho[TB];
        float w[TB];
        f32x4 t[TB];
#pragma unroll
        for (int b = 0; b < TB; ++b) {
          const int tok = b * 16 + l16;
          const bool mine = (tokens >> tok) & 1;
          const int r = (int)ex.first + __popcll(tokens & ((1ull << tok) - 1));
          ho[b] = mine ? (uint32_t)r * (uint32_t)c.I * 2u : kNowhere;
          w[b] = mine ? c.gate_of[(size_t)ex.id * kMaxTokens + tok] : 0.f;
          t[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        for (int s = wave * U; s < steps; s += kWaves * U) {
          typename Rows::Step fd[U];
#pragma unroll
          for (int u = 0; u < U; ++u) wd.load(fd[u], s + u, lane, s + u < steps);
#pragma unroll
          for (int b = 0; b < TB; ++b)
            if (TB == 1 || ((tokens >> (b * 16)) & 0xFFFFull) != 0) {
#pragma unroll
              for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t k = (uint32_t)(s + u) * 128u + Rows::column(i, g);
                  const u32x4 h = load16(rh, k < (uint32_t)c.I ? ho[b] + k * 2u : kNowhere);
                  t[b] = mfma_bf16(Rows::operand(fd[u], i), h, t[b]);
                }
            }
        }
        // a token that did not pick this expert adds nothing, whatever the weights hold
#pragma unroll
        for (int b = 0; b < TB; ++b)
          if (ho[b] != kNowhere) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[b][i] = __builtin_fmaf(w[b], t[b][i], y[b][i]);
          }
      }
#pragma unroll
      for (int b = 0; b < TB; ++b) partial[wave][b][lane] = y[b];
      __syncthreads();
      const int row = row0 + g * 4, tok = wave * 16 + l16;  // H is a multiple of 8
      const bool mine = wave < TB && tok < c.T && row < c.H;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (mine) {
        v = partial[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = v + partial[w][wave][lane];
      }
      bool store = mine;
      if (segments > 1) {
        float *out = c.sums + ((size_t)seg * c.T + tok) * c.H + row;
        if (mine) {
#pragma unroll
          for (int i = 0; i < 4; ++i) put_device(out + i, v[i]);
        }
        stores_done();
        if (threadIdx.x == 0) last = add_device(c.joined + rb) + 1 == (uint32_t)segments;
        __syncthreads();
        store = mine && last;
        if (store) {
          const float *in = c.sums + (size_t)tok * c.H + row;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = get_device(in + i);
          for (int s = 1; s < segments; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] + get_device(in + (size_t)s * c.T * c.H + i);
        }
      }
      if (store) {
        typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
        u32x2_e2 o;
        o[0] = pack_bf16(v[0], v[1]);
        o[1] = pack_bf16(v[2], v[3]);
        *reinterpret_cast<u32x2_e2 *>(c.y + (size_t)tok * c.ld_y + row) = o;
      }
    }
    if (threadIdx.x == 0) ticket = next;
    __syncthreads();  // `partial` and `last` are read, `ticket` is written
    task = ticket;
    __syncthreads();
  }
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// The workspace's parts; the counters come first.
struct MoeLayout {
  size_t plan, token_of, gate_of, joined, part, hidden, sums, end;
  int slices, segments, row_blocks;
};
MoeLayout layout_of(int T, int H, int I, int E, int k) {
  MoeLayout l{};
  // slices of H: a router workgroup's 8 waves take 128 columns each at a time
  l.slices = std::max(1, std::min(16, (H + 1023) / 1024));
  l.row_blocks = (H + 15) / 16;
  l.segments = std::max(1, std::min(std::min(E, T * k), (1024 + l.row_blocks - 1) / l.row_blocks));
  size_t at = up16(sizeof(MoeCounters));
  l.plan = at, at += up16((size_t)E * sizeof(MoeExpert));
  l.token_of = at, at += up16((size_t)T * k * 4);
  l.gate_of = at, at += up16((size_t)E * kMaxTokens * 4);
  l.joined = at, at += up16((size_t)l.row_blocks * 4);
  l.part = at, at += up16((size_t)l.slices * T * E * 4);
  l.hidden = at, at += up16((size_t)T * k * I * 2);
  l.sums = at, at += up16(l.segments > 1 ? (size_t)l.segments * T * H * 4 : 0);
  l.end = at;
  return l;
}

typedef void (*MoeFn)(MoeCall);
template <bool MX>
MoeFn experts_fn(int tb) {
  return tb == 1 ? moe_experts_kernel<MX, 1> : tb == 2 ? moe_experts_kernel<MX, 2> : moe_experts_kernel<MX, 4>;
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
  c.token_of = reinterpret_cast<int *>(ws + l.token_of);
  c.gate_of = reinterpret_cast<float *>(ws + l.gate_of);
  c.joined = reinterpret_cast<uint32_t *>(ws + l.joined);
  c.part = reinterpret_cast<float *>(ws + l.part);
  c.hidden = reinterpret_cast<uint16_t *>(ws + l.hidden);
  c.sums = reinterpret_cast<float *>(ws + l.sums);
  const int tb = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
  const MoeFn route = tb == 1 ? moe_route_kernel<1> : tb == 2 ? moe_route_kernel<2> : moe_route_kernel<4>;
  hipLaunchKernelGGL(route, dim3((a.experts + 15) / 16 * l.slices), dim3(kThreads), 0, s, c);
  if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  hipLaunchKernelGGL(mx ? experts_fn<true>(tb) : experts_fn<false>(tb), dim3(di->num_cus * 2), dim3(kThreads), 0, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int validate_moe_sizes(int T, int H, int I, int E, int k) {
  if (T < 0 || T > kMaxTokens || E < 1 || E > kMaxExperts || k < 1 || k > kMaxTopK || k > E) return OCC_EINVAL;
  if (H < 8 || H > 65536 || H % 8 != 0 || I < 8 || I > 65536 || I % 8 != 0) return OCC_EINVAL;
  return OCC_OK;
}

}  // namespace occ
