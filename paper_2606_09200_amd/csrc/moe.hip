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
//
// 64 tokens, 32 experts of 4096 x 2048 bf16, top 4: 277 us, 5.8 TB/s (16 for the router, 167 and 93 for the
// products, 6.4 and 5.8 TB/s).  37 tokens, 60 of 2504 x 1400: 227 us (12, 142, 73; 5.0 TB/s).  One token, 8
// of 64 experts of 4096 x 2048: MX4 40 us (9, 18, 12; 3.9 and 3.0 TB/s), latency; bf16 82 (9, 49, 24; 5.6 TB/s).
// 64 tokens, 32 of them MX4: 142 us (16, 72, 54; 4.0 and 2.6 TB/s).
#include "block_util.h"
#include "moe_extent.h"
#include "mx4.h"
#include "once.h"

#include <algorithm>
#include <cmath>

namespace occ {
namespace {

constexpr int kMaxTokens = 64, kMaxTopK = 16, kMaxExperts = 512, kMaxDevices = 64;
constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr uint32_t kNowhere = 0x80000000u;  // a byte offset beyond every descriptor

// 16 bytes at `off` (checked against the descriptor's end) plus `uniform` (which stays within a row).
template <int POLICY = 0>
__device__ __forceinline__ u32x4 load16(__amdgpu_buffer_rsrc_t r, uint32_t off, uint32_t uniform = 0) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)uniform, POLICY);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00020000);
}

template <class V>
__device__ __forceinline__ void put_device(V *p, V v) {  // through the XCD's L2, for readers on other XCDs
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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

// Largest of 32-bit words over a wave, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
  const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(s[0], s[1]);
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(t[0], t[1]);
}

// ---------------------------------------------------------------------------
// Router.  A workgroup multiplies 16 experts' rows with all tokens over one of `slices`
// slices of H, a wave 16 tokens and 128 columns at a time; the partial logits go to
// part[16 experts, slice][token][expert].  The workgroup that arrives last adds the slices in
// order, all tokens at once (they come from other XCDs' writes through memory), and picks:
// a wave per token at a time, lane l holding experts l, l + 64, ... (PER of them).
// Logits order as integers, a NaN below everything (its
// token's weights become NaN with the sum); equal ones go to the lower index.
//
// What bounds it is latency: two trips to memory and one workgroup's tail.  Most of
// that workgroup's instructions run once and come from memory too (80 ns per 64
// bytes), so its loops stay rolled.
constexpr int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64, kSlices = 8;

template <int TB, int PER>
__global__ __launch_bounds__(kRouteThreads) void moe_route_kernel(MoeCall c) {
  __shared__ f32x4 partial[kRouteWaves / TB][TB][64];
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
    constexpr int STEPS = kRouteWaves / TB;
    const int e0 = eb * 16, rows = min(16, c.E - e0), t = wave % TB * 16 + l16;
    const auto rw = rsrc_of(c.router + (size_t)e0 * c.H, (uint32_t)rows * (uint32_t)c.H * 2u);
    const auto rx = rsrc_of(c.x, ((uint32_t)(c.T - 1) * (uint32_t)c.ld_x + (uint32_t)c.H) * 2u);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const int steps = (c.H + 127) / 128;
#pragma unroll 1
    for (int s = slice * STEPS + wave / TB; s < steps; s += c.slices * STEPS) {
      u32x4 w[4], x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t k = (uint32_t)(s * 128 + i * 32 + g * 8);
        const bool in = k < (uint32_t)c.H;
        w[i] = load16(rw, in ? ((uint32_t)l16 * (uint32_t)c.H + k) * 2u : kNowhere);
        x[i] = load16(rx, in && t < c.T ? ((uint32_t)t * (uint32_t)c.ld_x + k) * 2u : kNowhere);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) acc = mfma_bf16(w[i], x[i], acc);
    }
    partial[wave / TB][wave % TB][lane] = acc;
    __syncthreads();
    // a thread per 4 experts (g) of a token
    if (threadIdx.x < TB * 64) {
      const int b = threadIdx.x >> 6, t = b * 16 + l16;
      f32x4 v = partial[0][b][lane];
#pragma unroll
      for (int w = 1; w < STEPS; ++w) v = v + partial[w][b][lane];
      if (t < c.T)
        __builtin_amdgcn_raw_buffer_store_b128(
            __builtin_bit_cast(u32x4, v), rsrc_of(c.part + (size_t)blockIdx.x * c.T * 16, (uint32_t)c.T * 64u),
            t * 64 + g * 16, 0, 16);  // device scope, as put_device
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
  extern __shared__ __align__(16) unsigned char smem[];
  float *logits = reinterpret_cast<float *>(smem);  // [token][pitch]
  const int pitch = (c.E + 15) / 16 * 16;
  {
    const auto rp = rsrc_of(c.part, (uint32_t)(pitch * c.slices * c.T) * 4u);
    const int per_block = c.T * 4;  // 16-byte pieces of 16 experts' logits
    for (int i = threadIdx.x; i < pitch * c.T / 4; i += kRouteThreads) {
      const int b = i / per_block, in = i % per_block;
      f32x4 part[kSlices];
#pragma unroll
      for (int s = 0; s < kSlices; ++s)
        if (s < c.slices)
          part[s] = __builtin_bit_cast(f32x4, load16<16>(rp, (uint32_t)((b * c.slices + s) * per_block + in) * 16u));
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSlices; ++s)
        if (s < c.slices) v = v + part[s];
      *reinterpret_cast<f32x4 *>(logits + (in >> 2) * pitch + b * 16 + (in & 3) * 4) = v;
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int t = wave; t < c.T; t += kRouteWaves) {
    const bool live = c.mask == nullptr || c.mask[t] != 0;
    float l[PER];
    uint32_t key[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      l[j] = j * 64 + lane < c.E ? logits[t * pitch + j * 64 + lane] : 0.f;
      // ascending integers, 1 and above; what is taken or missing is 0
      const uint32_t u = __builtin_bit_cast(uint32_t, l[j]);
      key[j] = j * 64 + lane >= c.E ? 0u : l[j] != l[j] ? 1u : (u >> 31 ? ~u : u | 0x80000000u);
    }
    float top = 0.f, mine = 0.f;  // mine: lane j < k holds pick j's logit, then its weight
    int my_id = 0;
#pragma unroll 1
    for (int j = 0; j < c.k; ++j) {
      uint32_t best = key[0];
#pragma unroll
      for (int i = 1; i < PER; ++i) best = max(best, key[i]);
      const uint32_t win = wave_max(best);
      int e = 0;  // the lowest index among equals
      float v = 0.f;
#pragma unroll
      for (int i = PER - 1; i >= 0; --i) {
        const uint64_t has = __ballot(key[i] == win);
        if (has != 0) {
          const int at = __builtin_ctzll(has);
          e = i * 64 + at;
          v = as_float((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, l[i]), at));
        }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i * 64 + lane == e) key[i] = 0u;
      if (j == 0) top = v;
      if (lane == j) mine = v, my_id = e;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum = sum + (i * 64 + lane < c.E ? expf(l[i] - top) : 0.f);
    sum = wave_sum(sum);
    float w = lane < c.k ? expf(mine - top) : 0.f;
    // a NaN among the logits is in `sum`, whichever experts were picked
    if (c.renorm) sum = sum == sum ? wave_sum(w) : sum;
    w = w / sum;
    if (lane < c.k) {
      if (!live) my_id = -1, w = 0.f;
      if (c.ids != nullptr) c.ids[t * c.k + lane] = my_id;
      if (c.weights != nullptr) c.weights[t * c.k + lane] = w;
      id_of[t][lane] = my_id;
      weight_of[t][lane] = w;
      if (live) atomicOr(&picked[my_id][t >> 5], 1u << (t & 31));
    }
  }
  __syncthreads();
  // active experts in index order, with the first of their rows of the hidden activations; one with
  // more than 32 tokens is two entries, whose weights are read twice
  const int e = threadIdx.x;
  const uint32_t m0 = e < c.E ? picked[e][0] : 0u, m1 = e < c.E ? picked[e][1] : 0u;
  const int n = __popc(m0) + __popc(m1);
  const uint64_t act = __ballot(n > 0), two = __ballot(n > 32);  // one or two entries of the list
  int before = n;  // pairs of lower lanes
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(before, d);
    if (lane >= d) before += o;
  }
  if (lane == 63) wave_pairs[wave] = before;
  if (lane == 0) wave_active[wave] = __popcll(act) + __popcll(two);
  before -= n;
  __syncthreads();
  int slot = __popcll(act & ((1ull << lane) - 1)) + __popcll(two & ((1ull << lane) - 1)), total = 0;
#pragma unroll
  for (int w = 0; w < kRouteWaves; ++w) {
    if (w < wave) slot += wave_active[w], before += wave_pairs[w];
    total += wave_active[w];
  }
  if (threadIdx.x == 0) c.count->active = total;
  if (n > 0) {
    c.plan[slot] = MoeExpert{(uint32_t)e, (uint32_t)before, (uint32_t)min(n, 32), 0u};
    if (n > 32) c.plan[slot + 1] = MoeExpert{(uint32_t)e, (uint32_t)before + 32u, (uint32_t)n - 32u, 0u};
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
// A 16-row block of an expert's matrix, read in units of 256 bytes a row of bf16 (128 columns) and
// 128 of MX4 (256 columns; the other factor's operands for more would halve the waves on a
// CU).  A load takes whole pieces of 4 or 8 rows, and the unit turns into operands through
// LDS of the wave's own (chunks of 16 bytes spread by row, no bank conflicts, no
// barriers): loads of 64 bytes from each of 16 rows, as an MFMA's operand lies in memory,
// are 10 % slower over the layer.  Where pieces are whole cache lines, each read once, the
// loads are non-temporal (one token, MX4: 55 -> 45 us; 64 tokens, bf16: 403 -> 360);
// where neighbouring pieces share lines that costs 8 % (rows of 2800 bytes).
//
// STEPS steps of 128 columns, each four MFMA operands of 32.  bf16: operand i of a step is
// columns 32 i + 8 g .. + 7 of lane (row, g).  MX4: a lane's 16 bytes are the block of columns
// 32 g .. + 31 of the step, operand i its columns 8 i .. + 7, converted to bf16 (exactly:
// E2M1 has two bits of precision) with the block's scale; the other factor is read
// in the same order.
template <bool MX>
struct Unit {
  u32x4 w[MX ? 2 : 4];  // load i: CH lanes to a row, rows 64 / CH apart
  uint32_t scale;       // MX4: the lane's word of the scale tile, its first two bytes the unit's steps
};

template <bool MX>
struct Rows16 {
  static constexpr int STEPS = MX ? 2 : 1, COLS = 128 * STEPS;
  static constexpr int CH = MX ? 8 : 16, LOADS = CH / 4;  // 16-byte chunks of a row, loads of a unit
  static constexpr int LDS = 16 * CH;                     // chunks of a staged unit
  __amdgpu_buffer_rsrc_t r, rs;
  uint32_t at, pitch, left;  // left: bytes of a row past the lane's first chunk
  bool whole;                // pieces are whole cache lines
  __device__ __forceinline__ Rows16(const MoeMatrix &m, int e, int row0, int rows, int cols, int lane) {
    pitch = MX ? (uint32_t)(OCC_MX4_KP(cols) / 2) : (uint32_t)cols * 2u;
    const MoeExtent w = moe_rows_extent(pitch, row0, rows), s = moe_scales_extent(pitch, row0, rows);
    r = rsrc_of(static_cast<const uint8_t *>(m.w) + (size_t)e * m.stride + w.at, w.bytes);
    if constexpr (MX) rs = rsrc_of(m.scales + (size_t)e * m.scale_stride + s.at, s.bytes);
    at = (uint32_t)(lane / CH) * pitch + (uint32_t)(lane % CH) * 16u;
    left = pitch - (uint32_t)(lane % CH) * 16u;
    whole = pitch % 128u == 0u && ((uintptr_t)m.w + m.stride) % 128u == 0u && m.stride % 128u == 0u;
  }
  __device__ __forceinline__ void load(Unit<MX> &q, int unit, int lane) const {
    const uint32_t k = (uint32_t)unit * (CH * 16u), step = 64u / CH * pitch;
    if (MX || (k + CH * 16u <= pitch && whole)) {  // MX4 rows are whole units
#pragma unroll
      for (int i = 0; i < LOADS; ++i) q.w[i] = load16<2>(r, at + i * step, k);
    } else if (k + CH * 16u <= pitch) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) q.w[i] = load16(r, at + i * step, k);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) q.w[i] = load16(r, (int)(left - k) > 0 ? at + i * step + k : kNowhere);
    }
    if constexpr (MX)  // a tile is two units; the second one's bytes are the upper half of its words
      q.scale = __builtin_amdgcn_raw_buffer_load_b16(rs, lane * 4, (int)((uint32_t)(unit >> 1) * 256u + (unit & 1) * 2u), 0);
  }
};

// Where chunk c of a row of a staged unit lies.
template <bool MX>
__device__ __forceinline__ int slot_of(int row, int c) {
  return MX ? row * 8 + swz<8>(row, c) : row * 16 + (c ^ row);
}
template <bool MX>
__device__ __forceinline__ void stage(u32x4 *lds, const Unit<MX> &q, int lane) {
  constexpr int CH = Rows16<MX>::CH;
#pragma unroll
  for (int i = 0; i < Rows16<MX>::LOADS; ++i) lds[slot_of<MX>(i * (64 / CH) + lane / CH, lane % CH)] = q.w[i];
}
// A lane's part of step s of a staged unit: operand i of bf16, or four operands' MX4 codes.
template <bool MX>
__device__ __forceinline__ u32x4 chunk(const u32x4 *lds, int i, int lane) {
  return lds[slot_of<MX>(lane & 15, 4 * i + (lane >> 4))];
}
// 8 MX4 codes with scale byte `s`.  The conversion takes the byte as a binary32 exponent: 0 is 2^-127, 255
// makes NaN (checked on every scale and code).
__device__ __forceinline__ u32x4 mx4_operand(uint32_t codes, uint32_t s) {
  const float sc = as_float(s << 23);
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 0));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 1));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 2));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 3));
  return o;
}

// The other factor's operands of a unit: rows (bf16) at byte offset `from` (kNowhere: none),
// which holds the lane's part already.
template <bool MX>
__device__ __forceinline__ uint32_t lane_bytes(int g) {
  return (MX ? 64u : 16u) * (uint32_t)g;
}
template <bool MX>
__device__ __forceinline__ void factor(u32x4 (&x)[Rows16<MX>::STEPS][4], __amdgpu_buffer_rsrc_t r, uint32_t from, int unit,
                                       int cols, int g) {
  constexpr uint32_t kNext = MX ? 16 : 64;  // bytes from operand to operand
  const uint32_t k = (uint32_t)unit * Rows16<MX>::COLS * 2u;
  if (k + Rows16<MX>::COLS * 2u <= (uint32_t)cols * 2u) {
#pragma unroll
    for (int s = 0; s < Rows16<MX>::STEPS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[s][i] = load16(r, from + 256u * s + kNext * i, k);
  } else {
    const uint32_t end = (uint32_t)cols * 2u - lane_bytes<MX>(g);
#pragma unroll
    for (int s = 0; s < Rows16<MX>::STEPS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t at = k + 256u * s + kNext * i;
        x[s][i] = load16(r, (int)(end - at) > 0 ? from + at : kNowhere);
      }
  }
}

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

// Two 16-row blocks times one unit of the other factor's columns, NB times 16 of them: acc0 += A x, acc1 += B x.
template <bool MX, int NB>
__device__ __forceinline__ void multiply(f32x4 *acc0, f32x4 *acc1, const u32x4 *lds, uint32_t scale0, uint32_t scale1,
                                         const u32x4 (*x)[Rows16<MX>::STEPS][4], int lane) {
  if constexpr (!MX) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 a = chunk<MX>(lds, i, lane), b = chunk<MX>(lds + Rows16<MX>::LDS, i, lane);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        acc0[n] = mfma_bf16(a, x[n][0][i], acc0[n]);
        acc1[n] = mfma_bf16(b, x[n][0][i], acc1[n]);
      }
    }
  } else {
#pragma unroll
    for (int s = 0; s < Rows16<MX>::STEPS; ++s) {
      const u32x4 a = chunk<MX>(lds, s, lane), b = chunk<MX>(lds + Rows16<MX>::LDS, s, lane);
      const uint32_t sa = scale0 >> (8 * s) & 255u, sb = scale1 >> (8 * s) & 255u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 wa = mx4_operand(a[i], sa), wb = mx4_operand(b[i], sb);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          acc0[n] = mfma_bf16(wa, x[n][s][i], acc0[n]);
          acc1[n] = mfma_bf16(wb, x[n][s][i], acc1[n]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // a step's operands at a time: registers
    }
  }
}

// A hidden activation h as two bf16 values, a row of each: h cut off after 8 bits, and what is left, rounded; together
// 15 bits or more.  Rounded to one bf16 value instead, y of every case of 1 to 64 tokens was off by 0.0023 of its size,
// with two by 0.0016, which is y's own rounding.  The second product takes as long up to 16 tokens and longer
// beyond (32 experts of 4096 x 2048: 24 tokens MX4 37 -> 40 us, 64 tokens MX4 39 -> 55, bf16 84 -> 93).
// The lower half has the upper one's sign and is not zero beside it (2^-24 of it instead), and an
// infinity or NaN is both: an infinite weight gives an infinity, as it does with h in one piece.
__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
}
__device__ __forceinline__ float lower_half(float h) {
  const float top = as_float(__builtin_bit_cast(uint32_t, h) & 0xFFFF0000u), r = h - top;
  return __builtin_fabsf(h) < __builtin_inff() ? (r == 0.f ? top * 0x1p-24f : r) : h;
}

// ---------------------------------------------------------------------------
// silu(Wg x) * (Wu x).  A task is `rbs` blocks of 16 rows of Wg and of Wu of one expert with that
// expert's tokens (16 to an MFMA).  8 / rbs waves split H (more blocks where H has fewer
// units than there are waves), the sums meet in LDS in wave order, and the result becomes
// two bf16 values, the next product's operands.
//
// What bounds it is the stream of weights, so it must not stop: a wave has the next
// unit's weights in flight while it multiplies (loads return in order: the other
// factor's are asked for before them), also across the end of a task, and two
// workgroups share a CU.  With AHEAD = 2 a wave has two units in flight: one workgroup a CU of
// them keeps up a stream of bf16 weights for many tokens better (64 tokens: 204 us, with it 180; 167 with
// up_row_blocks()'s four blocks a task), and two of them MX4's for few.
template <bool MX, int TB, int AHEAD>
__global__ __launch_bounds__(kThreads, !MX && AHEAD > 1 ? 2 : 4) void moe_up_kernel(MoeCall c) {
  typedef Rows16<MX> Rows;
  // a wave's units of Wg and Wu; its sums at the end of a task
  constexpr int AREA = 2 * Rows::LDS > 128 * TB ? 2 * Rows::LDS : 128 * TB;
  __shared__ u32x4 staged[kWaves][AREA];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  u32x4 *lds = staged[wave];
  const int kws = kWaves / c.rbs;           // waves along H
  const int kw = wave % kws, rsub = wave / kws;
  const uint32_t groups = (uint32_t)(c.I + 16 * c.rbs - 1) / (uint32_t)(16 * c.rbs);
  // the first task's expert is read beside the number of tasks, not after it
  MoeExpert ex = expert_at(c, min(blockIdx.x / groups, (uint32_t)(c.E * (c.T > 32 ? 2 : 1)) - 1u));
  const uint32_t tasks = __builtin_amdgcn_readfirstlane(c.count->active) * groups;
  if (blockIdx.x >= tasks) return;
  const auto rx = rsrc_of(c.x, ((uint32_t)(c.T - 1) * (uint32_t)c.ld_x + (uint32_t)c.H) * 2u);
  const int units = (c.H + Rows::COLS - 1) / Rows::COLS;
  const int u0 = kw, u1 = units;  // every kws-th, so that the waves together read whole rows
  auto row_of = [&](uint32_t task) { return moe_block_row((int)(task % groups) * c.rbs * 16, rsub, c.I); };
  Unit<MX> wg[AHEAD], wu[AHEAD];
  struct Cursor {  // the unit to load next
    uint32_t task;
    int expert, row0, u;
  } cur{blockIdx.x, (int)ex.id, row_of(blockIdx.x), u0};
  auto load = [&](Unit<MX> &qg, Unit<MX> &qu) {
    if (cur.task >= tasks || u0 >= u1) return;
    Rows(c.gate, cur.expert, cur.row0, c.I, c.H, lane).load(qg, cur.u, lane);
    Rows(c.up, cur.expert, cur.row0, c.I, c.H, lane).load(qu, cur.u, lane);
    cur.u += kws;
    if (cur.u >= u1) {
      cur.task += gridDim.x;
      if (cur.task < tasks) cur.expert = (int)expert_at(c, cur.task / groups).id;
      cur.row0 = row_of(cur.task);
      cur.u = u0;
    }
  };
  auto from_of = [&](const MoeExpert &e, int at) {  // where the lane's token of the at-th 16 lies
    return at * 16 + l16 < (int)e.n
               ? (uint32_t)c.rows[e.first + at * 16 + l16].token * (uint32_t)c.ld_x * 2u + lane_bytes<MX>(g) : kNowhere;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(wg[i], wu[i]);
  int slot = 0;
  uint32_t xo = from_of(ex, 0);
#pragma unroll 1
  for (uint32_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const uint32_t nxt = task + gridDim.x;
    const MoeExpert en = nxt < tasks ? expert_at(c, nxt / groups) : ex;
    const int n = (int)ex.n, nb = (n + 15) / 16;
    const uint32_t xn = from_of(en, 0);
    f32x4 ag[TB], au[TB];
#pragma unroll
    for (int at = 0; at < TB; ++at) ag[at] = au[at] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int u = u0; u < u1; u += kws) {
      u32x4 x[1][Rows::STEPS][4];
      factor<MX>(x[0], rx, xo, u, c.H, g);
      // this unit's weights leave the registers, the next one's are on their way into them
      uint32_t sg, su;
      auto turn = [&](Unit<MX> &qg, Unit<MX> &qu) {
        sg = qg.scale, su = qu.scale;
        stage<MX>(lds, qg, lane);
        stage<MX>(lds + Rows::LDS, qu, lane);
        __builtin_amdgcn_sched_barrier(0);
        load(qg, qu);
        __builtin_amdgcn_sched_barrier(0);
      };
      if (AHEAD == 1 || slot == 0) turn(wg[0], wu[0]);
      else turn(wg[AHEAD - 1], wu[AHEAD - 1]);
      if (AHEAD > 1) slot ^= 1;
      multiply<MX, 1>(&ag[0], &au[0], lds, sg, su, x, lane);
#pragma unroll
      for (int at = 1; at < TB; ++at)
        if (at < nb) {
          factor<MX>(x[0], rx, from_of(ex, at), u, c.H, g);
          multiply<MX, 1>(&ag[at], &au[at], lds, sg, su, x, lane);
        }
    }
    f32x4 *sums = reinterpret_cast<f32x4 *>(lds);  // [16 tokens][Wg, Wu][lane]
#pragma unroll
    for (int at = 0; at < TB; ++at)
      if (at < nb) {
        sums[at * 128 + lane] = ag[at];
        sums[at * 128 + 64 + lane] = au[at];
      }
    __syncthreads();
    // wave: 16 rows of the task and 16 tokens
    for (int v = wave; v < c.rbs * nb; v += kWaves) {
      const int rs = v % c.rbs, at = v / c.rbs;
      const f32x4 *in = reinterpret_cast<const f32x4 *>(staged[rs * kws]) + at * 128 + lane;
      f32x4 gs = in[0], us = in[64];
      for (int w = 1; w < kws; ++w) {
        gs = gs + in[w * AREA];
        us = us + in[w * AREA + 64];
      }
      float h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = gs[i] / (1.f + expf(-gs[i])) * us[i];
      const int row = ((int)(task % groups) * c.rbs + rs) * 16 + g * 4;  // I is a multiple of 8: all four exist or none
      if (at * 16 + l16 < n && row < c.I) {
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = lower_half(h[i]);
        uint16_t *to = c.hidden + (size_t)(ex.first + at * 16 + l16) * 2 * c.I + row;
        *reinterpret_cast<uint64_t *>(to) = (uint64_t)upper_halves(h[2], h[3]) << 32 | upper_halves(h[0], h[1]);
        *reinterpret_cast<uint64_t *>(to + c.I) = (uint64_t)pack_bf16(r[2], r[3]) << 32 | pack_bf16(r[0], r[1]);
      }
    }
    __syncthreads();  // before the sums' place is staged into again
    ex = en;
    xo = xn;
  }
}

// ---------------------------------------------------------------------------
// y = sum_j w_j Wd_j h_j.  A task is 32 rows of Wd for the experts of one of `segments` parts
// of the list; the waves split those experts' columns end to end, each adding its
// experts' weighted sums to its own rows of y in LDS, one per token (a token that did not
// pick an expert gets nothing from it, whatever its weights hold).  An activation's two halves are
// neighbouring columns of a 16-column block, up to TB of them, and their lanes add up at the end.  With several segments
// the last one to finish a block of rows adds them in order: no sum depends on timing.
// The weights' stream is kept up as above; a cursor runs AHEAD units in front of the
// multiplications, across experts and tasks.  AHEAD is 2 where a CU has one workgroup.
template <bool MX, int TB, int AHEAD>
__global__ __launch_bounds__(kThreads, AHEAD == 1 ? 4 : 2) void moe_down_kernel(MoeCall c) {
  typedef Rows16<MX> Rows;
  __shared__ u32x4 staged[kWaves][2 * Rows::LDS];        // a wave's units of the two row blocks
  extern __shared__ __align__(16) unsigned char smem[];  // y: [wave][token][32 rows]
  constexpr int XA = TB > 1 ? 2 : 1;  // blocks of 16 columns asked for ahead of the next weights
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  u32x4 *lds = staged[wave];
  const int active = (int)__builtin_amdgcn_readfirstlane(c.count->active);
  const int segments = max(1, min(active, c.max_segments));
  const int tasks = c.row_blocks * segments;
  if ((int)blockIdx.x >= tasks) return;
  const auto rh = rsrc_of(c.hidden, (uint32_t)(c.T * c.k) * (uint32_t)c.I * 4u);
  const int units = (c.I + Rows::COLS - 1) / Rows::COLS;  // of one expert
  Unit<MX> w0[AHEAD], w1[AHEAD];
  // Of a task: its rows, its first expert, and this wave's units of all its experts, end to end, from
  // `start` round.  Long tasks start at different columns: with all at the same ones, and rows a power of
  // two apart, only some of the memory's channels answer (64 tokens, 32 experts of 4096 x 2048
  // bf16 in tasks of 16 experts: 113 us, now 84).  It gains nothing with MX4's shorter rows.
  struct Part {
    int row0, a0, u0, u1, start;
  };
  auto part_of = [&](int task) {
    const int seg = task % segments;
    Part p;
    p.row0 = task / segments * 32;
    p.a0 = seg * active / segments;
    const int all = ((seg + 1) * active / segments - p.a0) * units;
    p.u0 = wave * all / kWaves;
    p.u1 = (wave + 1) * all / kWaves;
    p.start = !MX && p.u1 - p.u0 >= 8 ? p.u0 + task / segments % (p.u1 - p.u0) : p.u0;
    return p;
  };
  struct Cursor {  // the unit to load next: `left` units of the task, unit `k` of list entry `a`
    int task, row0, left, to_end, a, k, a0, k0;
  } cur;
  auto enter = [&](int task) {  // the first task from this one on in which the wave has a unit
    cur.left = 0;
    for (; task < tasks && cur.left == 0; task += gridDim.x) {
      const Part p = part_of(task);
      cur.task = task, cur.row0 = p.row0, cur.left = p.u1 - p.u0;
      cur.to_end = p.u1 - p.start;
      cur.a = p.a0 + p.start / units, cur.k = p.start % units;
      cur.a0 = p.a0 + p.u0 / units, cur.k0 = p.u0 % units;
    }
  };
  auto load = [&](Unit<MX> &q0, Unit<MX> &q1) {
    if (cur.left == 0) return;
    const int e = (int)expert_at(c, cur.a).id;
    Rows(c.down, e, cur.row0, c.H, c.I, lane).load(q0, cur.k, lane);
    Rows(c.down, e, moe_block_row(cur.row0, 1, c.H), c.H, c.I, lane).load(q1, cur.k, lane);
    if (++cur.k == units) cur.k = 0, ++cur.a;
    if (--cur.to_end == 0) cur.a = cur.a0, cur.k = cur.k0;
    if (--cur.left == 0) enter(cur.task + gridDim.x);
  };
  enter(blockIdx.x);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(w0[i], w1[i]);
  int slot = 0;
  float *y = reinterpret_cast<float *>(smem), *mine = y + wave * c.T * 32;
#pragma unroll 1
  for (int task = blockIdx.x; task < tasks; task += gridDim.x) {
    const Part p = part_of(task);
    for (int i = lane; i < c.T * 8; i += 64) reinterpret_cast<f32x4 *>(mine)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int u = p.start, left = p.u1 - p.u0; left > 0;) {
      const MoeExpert ex = expert_at(c, p.a0 + u / units);
      const int n = 2 * (int)ex.n, nb = (n + 15) / 16;  // columns: an activation's two halves
      const int end = min(min(p.u1, (u / units + 1) * units), u + left);
      left -= end - u;
      auto from_of = [&](int at) {
        return at * 16 + l16 < n ? (2 * ex.first + at * 16 + l16) * (uint32_t)c.I * 2u + lane_bytes<MX>(g) : kNowhere;
      };
      f32x4 a0[TB], a1[TB];
      MoeRow row[TB];
#pragma unroll
      for (int at = 0; at < TB; ++at) {
        a0[at] = a1[at] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (at * 16 + l16 < n) row[at] = c.rows[ex.first + (at * 16 + l16) / 2];
      }
#pragma unroll 1
      for (; u < end; ++u) {
        u32x4 x[XA][Rows::STEPS][4];
#pragma unroll
        for (int at = 0; at < XA; ++at)
          if (at < nb) factor<MX>(x[at], rh, from_of(at), u % units, c.I, g);
        uint32_t s0, s1;
        auto turn = [&](Unit<MX> &q0, Unit<MX> &q1) {
          s0 = q0.scale, s1 = q1.scale;
          stage<MX>(lds, q0, lane);
          stage<MX>(lds + Rows::LDS, q1, lane);
          __builtin_amdgcn_sched_barrier(0);
          load(q0, q1);
          __builtin_amdgcn_sched_barrier(0);
        };
        if (AHEAD == 1 || slot == 0) turn(w0[0], w1[0]);
        else turn(w0[AHEAD - 1], w1[AHEAD - 1]);
        if (AHEAD > 1) slot ^= 1;
        if (XA == 1 || nb == 1) multiply<MX, 1>(&a0[0], &a1[0], lds, s0, s1, x, lane);
        else multiply<MX, XA>(&a0[0], &a1[0], lds, s0, s1, x, lane);
        if (TB > 2 && nb > 2) {
#pragma unroll
          for (int at = 0; at < XA; ++at) factor<MX>(x[at], rh, from_of(XA + at), u % units, c.I, g);
          multiply<MX, XA>(&a0[TB - XA], &a1[TB - XA], lds, s0, s1, x, lane);
        }
      }
      if (u == p.u1) u = p.u0;
      // this part of the expert is whole: into its tokens' rows
#pragma unroll
      for (int at = 0; at < TB; ++at)
        if (at * 16 + l16 < n) {
          // both halves' lanes have both sums; the upper's takes the first 16 rows, the lower's the others
          f32x4 *to = reinterpret_cast<f32x4 *>(mine + row[at].token * 32 + (l16 & 1) * 16 + g * 4);
          f32x4 v = *to;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float s0 = a0[at][i] + dpp<0xB1>(a0[at][i]), s1 = a1[at][i] + dpp<0xB1>(a1[at][i]);
            v[i] = __builtin_fmaf(row[at].weight, l16 & 1 ? s1 : s0, v[i]);
          }
          *to = v;
        }
    }
    __syncthreads();
    const int rb = task / segments, seg = task % segments;
    const int tok = threadIdx.x >> 3, row = p.row0 + (threadIdx.x & 7) * 4;  // H is a multiple of 8
    const bool has = tok < c.T && row < c.H;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (has) {
      const f32x4 *in = reinterpret_cast<const f32x4 *>(y) + threadIdx.x;
      v = in[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v = v + in[w * c.T * 8];
    }
    bool store = has;
    if (segments > 1) {
      constexpr int kDevice = 16;  // cache policy: device scope, as put_device
      const uint32_t at = ((uint32_t)tok * (uint32_t)c.H + (uint32_t)row) * 4u, whole = (uint32_t)c.T * (uint32_t)c.H * 4u;
      const auto rs = rsrc_of(c.sums, whole * (uint32_t)segments);
      if (has) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, (int)(seg * whole + at), 0, kDevice);
      stores_done();
      uint32_t *last = reinterpret_cast<uint32_t *>(y);  // y has been read
      if (threadIdx.x == 0) *last = add_device(c.joined + rb) + 1 == (uint32_t)segments;
      __syncthreads();
      store = has && *last != 0u;
      if (store) {
        v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < segments; ++s)
          v = v + __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(s * whole + at), 0, kDevice));
      }
    }
    if (store) {
      typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2)));
      u32x2_e2 o;
      o[0] = pack_bf16(v[0], v[1]);
      o[1] = pack_bf16(v[2], v[3]);
      *reinterpret_cast<u32x2_e2 *>(c.y + (size_t)tok * c.ld_y + row) = o;
    }
    __syncthreads();  // before y is cleared for the next task
  }
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// Experts that T tokens pick, on average.
double expected_active(int T, int E, int k) { return E * (1 - std::pow(1 - (double)k / E, T)); }

// Blocks of 16 rows in a task of the first product, whose waves split H between them: more where H has fewer
// units than there are waves.  Beside that, four with many bf16 tokens, which have one workgroup a CU, for
// fewer ends of tasks, where two rounds of such tasks are left (64 tokens, 32 experts of 4096 x
// 2048: 177 us, now 167; 2504 x 2048: 141, 126; 16 experts of 4096 x 4096 lose: 181, 187), and two
// with MX4 where every workgroup has a task (one token, 8 of 64 experts of 4096 x 2048: 17.9 us,
// now 16.4; 64 tokens: 122, 113).
int up_row_blocks(int T, int H, int I, int E, int k, bool mx, int workgroups) {
  const int units = mx ? (H + 255) / 256 : (H + 127) / 128, least = units >= 8 ? 1 : units >= 4 ? 2 : units >= 2 ? 4 : 8;
  const double active = expected_active(T, E, k);
  if (!mx) return T > 16 && active * ((I + 63) / 64) >= 1.9 * workgroups ? std::max(least, 4) : least;
  return active * ((I + 31) / 32) >= 0.95 * workgroups ? std::max(least, 2) : least;
}

// Workgroups of the second product on a CU: y of every wave is in LDS beside what its units pass through.
// Beyond 16 tokens with bf16 weights and 48 with MX4 that leaves room for one; beyond 8, an expert's tokens may be
// more than one block of 16 columns, whose operands do not fit in half a CU's registers (14 spilled).
int down_per_cu(int T) { return T <= 8 ? 2 : 1; }

// Parts of the list of experts that the second product's tasks take: the split of the least estimated
// time.  A task costs 2 us beside its units, 3 where parts have to be joined, and eight units (one a
// wave) what 32 rows of 512 bytes a wave take at a CU's share of 6 TB/s; tasks run in rounds of
// as many as the chip holds.  (Four tasks a workgroup whatever the sizes: 55 tokens of 8 experts, 6144 x
// 1264 MX4, 35 us, now 16; 37 tokens of 60 experts, 2504 x 1400 bf16, 93 us, now 69.)
int down_segments(int T, int H, int I, double active, int most, bool mx) {
  // 256 CUs, whatever the device: the workspace's size follows from the split and is asked for without one
  const double slots = 256.0 * down_per_cu(T), per_slot = 1 / slots;
  const int blocks = (H + 31) / 32, units = mx ? (I + 255) / 256 : (I + 127) / 128;
  const double unit_us = (mx ? 1.4 : 2.8) * down_per_cu(T), work = std::max(1.0, active) * units / kWaves;
  int best = 1;
  double t_best = 0;
  // past the last split that leaves a wave a unit, or four rounds of tasks, nothing is gained
  for (int seg = 1; seg <= most && (seg == 1 || (seg <= active && work >= seg && blocks * seg <= 4 * slots)); ++seg) {
    const double us = std::ceil(blocks * seg * per_slot) * ((seg > 1 ? 3 : 2) + unit_us * std::max(1.0, work / seg));
    if (seg == 1 || us < t_best) best = seg, t_best = us;
  }
  return best;
}

// The workspace's parts; the counters come first.
struct MoeLayout {
  size_t plan, rows, joined, part, hidden, sums, end;
  int slices, row_blocks, segments[2];  // of the second product with bf16 and with MX4 weights
};
MoeLayout layout_of(int T, int H, int I, int E, int k) {
  MoeLayout l{};
  const int steps = kRouteWaves / (T <= 16 ? 1 : T <= 32 ? 2 : 4);  // of 128 columns, that a router workgroup takes at once
  l.slices = std::max(1, std::min(kSlices, (H + 128 * steps - 1) / (128 * steps)));
  l.row_blocks = (H + 31) / 32;
  const double active = expected_active(T, E, k);
  for (int mx = 0; mx < 2; ++mx) l.segments[mx] = down_segments(T, H, I, active, std::min(E, T * k), mx != 0);
  const int segments = std::max(l.segments[0], l.segments[1]);
  size_t at = up16(sizeof(MoeCounters));
  l.plan = at, at += up16((size_t)E * (T > 32 ? 2 : 1) * sizeof(MoeExpert));
  l.rows = at, at += up16((size_t)T * k * sizeof(MoeRow));
  l.joined = at, at += up16((size_t)l.row_blocks * 4);
  l.part = at, at += up16((size_t)l.slices * ((E + 15) / 16) * T * 64);
  l.hidden = at, at += up16((size_t)T * k * I * 4);
  l.sums = at, at += up16(segments > 1 ? (size_t)segments * T * H * 4 : 0);
  l.end = at;
  return l;
}

typedef void (*MoeFn)(MoeCall);
template <int PER>
MoeFn route_fn(int tb) {
  return tb == 1 ? moe_route_kernel<1, PER> : tb == 2 ? moe_route_kernel<2, PER> : moe_route_kernel<4, PER>;
}
MoeFn up_fn(bool mx, int tb) {
  if (mx) return tb == 1 ? moe_up_kernel<true, 1, 2> : moe_up_kernel<true, 2, 1>;
  return tb == 1 ? moe_up_kernel<false, 1, 1> : moe_up_kernel<false, 2, 2>;
}
template <bool MX>
MoeFn down_fn(int tokens) {
  return tokens <= 8 ? moe_down_kernel<MX, 1, 1> : tokens <= 16 ? moe_down_kernel<MX, 2, 2> : moe_down_kernel<MX, 4, 2>;
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
  c.slices = l.slices, c.row_blocks = l.row_blocks, c.max_segments = l.segments[a.weight_type == OCC_MX4];
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
  const int per = a.experts <= 64 ? 0 : a.experts <= 128 ? 1 : 2;
  const MoeFn route = per == 0 ? route_fn<1>(tb) : per == 1 ? route_fn<2>(tb) : route_fn<8>(tb);
  const int logits = a.tokens * ((a.experts + 15) / 16 * 16) * 4;
  // with the kernel's own 30 KB past what a launch may have unasked; the limit is the kernel's for all host threads, so
  // it is what any call needs
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return OCC_ENODEV;
  static Once limit_set[kMaxDevices][3][3];
  if (!limit_set[dev][per][tb >> 1].run([&] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(route), hipFuncAttributeMaxDynamicSharedMemorySize,
                                   kMaxTokens * kMaxExperts * 4) == hipSuccess;
      }))
    return OCC_EHIP;
  hipLaunchKernelGGL(route, dim3((a.experts + 15) / 16 * l.slices), dim3(kRouteThreads), logits, s, c);
  if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  const unsigned grid = (unsigned)di->num_cus * (!mx && tb > 1 ? 1 : 2);
  c.rbs = up_row_blocks(a.tokens, a.H, a.I, a.experts, a.top_k, mx, (int)grid);
  hipLaunchKernelGGL(up_fn(mx, tb), dim3(grid), dim3(kThreads), 0, s, c);
  if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  const int y_bytes = kWaves * a.tokens * 128, per_cu = down_per_cu(a.tokens);
  hipLaunchKernelGGL(mx ? down_fn<true>(a.tokens) : down_fn<false>(a.tokens), dim3(di->num_cus * per_cu), dim3(kThreads), y_bytes, s, c);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

int validate_moe_sizes(int T, int H, int I, int E, int k) {
  if (T < 0 || T > kMaxTokens || E < 1 || E > kMaxExperts || k < 1 || k > kMaxTopK || k > E) return OCC_EINVAL;
  if (H < 8 || H > 65536 || H % 8 != 0 || I < 8 || I > 65536 || I % 8 != 0) return OCC_EINVAL;
  return OCC_OK;
}

}  // namespace occ
