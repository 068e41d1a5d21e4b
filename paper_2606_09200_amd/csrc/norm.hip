// The norms after and before a block with its gate and the residual's scale
// (occ_norm_gate) and the gradients (occ_norm_gate_bwd).
//
//   n = f r1 w1, r1 = rsqrt(mean f^2 + eps);  y = alpha x + g n;  h = y r2 w2, r2 = rsqrt(mean y^2 + eps)
//
// and with u = dh w2:
//   D = dy + r2 u - y r2^3 mean(u y);  dx = alpha D;  df = r1 v - f r1^3 mean(v f), v = D g w1
//   S = sum D f r1 over the rows of a gate;  dg = w1 S;  dw1 = sum g S;  dw2 = sum dh y r2
//
// Both are bound by the bytes of the rows they read and write once; a row stays in
// registers between its two sums.  Sums, statistics and gradients of the
// parameters are binary32; rows are rounded once, when stored.  h is made from the unrounded y, while the gradients
// read y as it is stored: with a bf16 residual they are those of a row that is off by up to 2^-8 of itself, the
// price of storing nothing beside y.
//
// A row is chunks of 8 columns.  One that ends inside a chunk leaves that chunk's 8 registers
// with its values by fours, twos and ones at fixed places (Chunks), which takes two more
// loads and stores of one lane and no selects.
//
// 8192 rows of 8192 bf16: forward 95 us (5.6 TB/s of what it must read and write), backward 153
// us with its sums joined (5.3 TB/s); binary32: 198 and 311 us (5.4, 5.2).  12004 ragged rows of 5003
// with a binary32 residual: 144 and 221 us (5.0, 4.9).  16 rows of 8192: 6.4 us, of which a
// launch is 2.3 and the rest the way through two sums.  Rows beyond 8192 columns go backward at
// 4.5 TB/s: one row a CU in flight, nothing fetched ahead.
#include "block_util.h"

#include <algorithm>

namespace occ {
namespace {

// Sum over a workgroup, which has a row; `slot` holds 16 floats that no one else uses before the
// next barrier but one.  The order of the sum is fixed.
__device__ __forceinline__ float row_sum(float v, float *slot) {
  v = wave_sum(v);
  const int waves = (int)blockDim.x >> 6;
  if (waves > 1) {
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slot[0];
    for (int w = 1; w < waves; ++w) v = v + slot[w];
  }
  return v;
}

// This thread's chunks of a row.  REST: D is no multiple of 8, and the last chunk has 4, 2 and 1
// values by the bits of D: in elements 0 to 3, 4 and 5, and 6.  The other elements are
// zeros and add nothing to a sum.
template <int NCH, bool REST>
struct Chunks {
  uint32_t at[NCH];
  bool in[NCH], end[NCH];
  int D;
  __device__ __forceinline__ explicit Chunks(int d) : D(d) {
    const uint32_t whole = (uint32_t)D & ~7u;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      at[c] = (c * blockDim.x + threadIdx.x) * 8;
      in[c] = at[c] < whole;
      end[c] = REST && at[c] == whole;
    }
  }
  // Keeps the offsets from being folded into 64-bit addresses of each tensor's chunks, which would live
  // across rows: the backward pass spilled them.
  __device__ __forceinline__ void fresh() {
#pragma unroll
    for (int c = 0; c < NCH; ++c) asm volatile("" : "+v"(at[c]));
  }
  template <class E>
  __device__ __forceinline__ void load(Raw8<E> &v, const E *row, int c) const {
    v.load(element(row, at[c]), in[c]);
    if (REST && end[c]) v.load_rest(element(row, at[c]), D);
  }
  // NT for the forward rows (8192 rows of 8192 bf16: 94 us, without 100); the backward pass's are
  // stored plainly (8192 rows of 8192 binary32: 324 us, with 355).
  template <bool NT, class E>
  __device__ __forceinline__ void store(E *row, int c, const float (&v)[8]) const {
    store8<NT>(element(row, at[c]), in[c], v);
    if (REST && end[c]) store_rest(element(row, at[c]), D, v);
  }
};
int chunks(int D) { return (D + 7) / 8; }

// ---------------------------------------------------------------------------
// Forward.  A workgroup of as many waves as a row needs at NCH chunks of 8 columns a thread (chunk c
// of thread t: columns 8 (c threads + t)) has one row; one wave needs no barrier.  As many
// workgroups as the chip holds, each walking rows, were slower: their rows go in step (12004 rows of
// 5120: 161 us, now 132; 16384 of 4096: 100, 94).
template <int NCH, bool REST, class ACT, class RES>
__global__ __launch_bounds__(1024) void norm_gate_kernel(NormFwd a) {
  __shared__ float slots[2][16];
  const Chunks<NCH, REST> cols(a.D);
  const float inv_d = 1.0f / (float)a.D;
  const ACT *w1 = static_cast<const ACT *>(a.w_post), *w2 = static_cast<const ACT *>(a.w_pre);
  const int row = blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const ACT *f = static_cast<const ACT *>(a.f) + (size_t)row * a.ld_f;
  const RES *x = static_cast<const RES *>(a.x) + (size_t)row * a.ld_x;
  RES *yo = static_cast<RES *>(a.y) + (size_t)row * a.ld_y;
  ACT *ho = static_cast<ACT *>(a.h) + (a.h != nullptr ? (size_t)row * a.ld_h : 0);
  const ACT *gate = static_cast<const ACT *>(a.gate);
  if (gate != nullptr) gate += (size_t)(row / a.rows_per_gate) * a.D;
  Raw8<ACT> fv[NCH];
  Raw8<RES> xv[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) cols.load(fv[c], f, c);
#pragma unroll
  for (int c = 0; c < NCH; ++c) cols.load(xv[c], x, c);
  float r1 = 1.f;
  if (a.post) {
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(fv[c].at(e), fv[c].at(e), ss);
    r1 = 1.0f / __builtin_sqrtf(row_sum(ss, slots[0]) * inv_d + a.eps);
  }
  float ss = 0.f;
  float y[NCH][8];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[c][e] = fv[c].at(e) * r1;
    if (w1 != nullptr) {
      Raw8<ACT> w;
      cols.load(w, w1, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[c][e] = y[c][e] * w.at(e);
    }
    if (gate != nullptr) {
      Raw8<ACT> w;
      cols.load(w, gate, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[c][e] = y[c][e] * w.at(e);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[c][e] = __builtin_fmaf(a.alpha, xv[c].at(e), y[c][e]);
      ss = __builtin_fmaf(y[c][e], y[c][e], ss);
    }
    cols.template store<true>(yo, c, y[c]);
  }
  float r2 = 1.f;
  if (a.h != nullptr) {
    r2 = 1.0f / __builtin_sqrtf(row_sum(ss, slots[1]) * inv_d + a.eps);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[c][e] = y[c][e] * r2;
      if (w2 != nullptr) {
        Raw8<ACT> w;
        cols.load(w, w2, c);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[c][e] = y[c][e] * w.at(e);
      }
      cols.template store<true>(ho, c, y[c]);
    }
  }
  if (a.rstd != nullptr && threadIdx.x == 0) {
    a.rstd[2 * (size_t)row] = r1;
    a.rstd[2 * (size_t)row + 1] = r2;
  }
}

// ---------------------------------------------------------------------------
// Backward.  A workgroup of as many waves as a row needs at NCH chunks of 8 columns a thread takes a
// run of rows and keeps the sums over them; the next row's loads are in flight while a
// row is worked on.
//
// Where gates are shared by many rows (or there is none), a run stays within one
// gate's rows: every per_gate-th of them, so that all runs together walk through memory (runs of
// neighbouring rows: 8192 x 8192 bf16 165 us instead of 153, binary32 324 and 311).  S and dw2's sum leave as one row each of the
// partial arrays; with several gates g S does too, as the first.  Where gates are not
// shared so (DIRECT), a run is every runs-th whole gate: at the end of each, dg is
// complete and stored, and g S goes into the run's sum of dw1, the first array's row.
//
// Up to 8192 columns (NCH = 1) the sums, the weights and two rows fit in registers, but for 4 or 5 a thread that
// binary32 rows spill with DIRECT.
// Beyond (NCH = 2, 1024 threads of 128 registers) the sums live in LDS, the
// binary32 weights come from the caches for each row, and rows are not fetched ahead.  bf16 weights,
// which stay, leave 13 to 16 registers spilled with DIRECT, and one without where the residual is binary32.
template <int N, bool LDS>
struct ColumnSums;  // N sums a thread
template <int N>
struct ColumnSums<N, false> {
  float v[N];
  __device__ __forceinline__ explicit ColumnSums(float *) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
};
template <int N>
struct ColumnSums<N, true> {
  float *at;  // this thread's words, 1024 apart: no bank conflicts, no barriers
  __device__ __forceinline__ explicit ColumnSums(float *base) : at(base + threadIdx.x) {
#pragma unroll
    for (int i = 0; i < N; ++i) set(i, 0.f);
  }
  __device__ __forceinline__ float get(int i) const { return at[i * 1024]; }
  __device__ __forceinline__ void set(int i, float x) { at[i * 1024] = x; }
};

template <int NCH, bool REST, class ACT, class RES, bool DIRECT>
__global__ __launch_bounds__(1024) void norm_gate_bwd_kernel(NormBwd a) {
  constexpr bool WIDE = NCH > 1;
  constexpr bool KEEP = !WIDE || sizeof(ACT) == 2;  // weights stay in registers
  __shared__ float slots[2][2][16];
  extern __shared__ __align__(16) unsigned char smem[];  // WIDE: two arrays of 8 NCH 1024 sums
  float *lds = reinterpret_cast<float *>(smem);
  const int D = a.D;
  const float inv_d = 1.0f / (float)D;
  int row_begin, row_end, gate_at;
  if (DIRECT) {
    gate_at = blockIdx.x;
    row_begin = gate_at * a.rows_per_gate;
    row_end = a.rows;
  } else {
    gate_at = blockIdx.x / a.per_gate;
    row_begin = gate_at * a.rows_per_gate + (int)(blockIdx.x % a.per_gate);
    row_end = (gate_at + 1) * a.rows_per_gate;
  }
  Chunks<NCH, REST> cols(D);
  const ACT *w_post = static_cast<const ACT *>(a.w_post), *w_pre = static_cast<const ACT *>(a.w_pre);
  const ACT *gate = static_cast<const ACT *>(a.gate);
  Raw8<ACT> w1[NCH], w2[NCH], gv[NCH];
  // loaded again for each row: what a null pointer leaves is cleared, or the last row's registers would stay live
  // (80 of them in scratch memory, now none: 4096 rows of 16384 binary32 546 us, now 354)
  auto load_gate = [&](int c) {
    if (!KEEP) gv[c] = Raw8<ACT>{};
    if (gate != nullptr) cols.load(gv[c], gate + (size_t)gate_at * D, c);
  };
  auto load_post = [&](int c) {
    if (!KEEP) w1[c] = Raw8<ACT>{};
    if (w_post != nullptr) cols.load(w1[c], w_post, c);
  };
  auto load_pre = [&](int c) {
    if (!KEEP) w2[c] = Raw8<ACT>{};
    if (w_pre != nullptr) cols.load(w2[c], w_pre, c);
  };
  auto post = [&](int c, int e) { return w_post != nullptr ? w1[c].at(e) : 1.f; };
  auto gated = [&](int c, int e) { return gate != nullptr ? gv[c].at(e) : 1.f; };
  auto fence = [&]() {  // keeps loads from being moved up to where their registers are not free yet
    if (WIDE) __builtin_amdgcn_sched_barrier(0);
  };
  // S: of the run, or (DIRECT) of the gate; dw1: DIRECT only
  ColumnSums<8 * NCH, WIDE && !DIRECT> s1(lds);
  ColumnSums<8 * NCH, WIDE> s2(lds + 8 * NCH * 1024);
  ColumnSums<8 * NCH, WIDE && DIRECT> dw1(lds);
  if (KEEP)
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      load_post(c);
      load_pre(c);
      if (!DIRECT) load_gate(c);
    }
  struct Rows {
    Raw8<ACT> f[NCH], dh[NCH];
    Raw8<RES> y[NCH], dy[NCH];
    float r1, r2;
  };
  auto fetch = [&](Rows &q, int row) {
    q.r1 = a.rstd[2 * (size_t)row];
    q.r2 = a.rstd[2 * (size_t)row + 1];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (a.dh != nullptr) {
        cols.load(q.y[c], static_cast<const RES *>(a.y) + (size_t)row * a.ld_y, c);
        cols.load(q.dh[c], static_cast<const ACT *>(a.dh) + (size_t)row * a.ld_dh, c);
      }
      cols.load(q.f[c], static_cast<const ACT *>(a.f) + (size_t)row * a.ld_f, c);
      if (a.dy != nullptr) cols.load(q.dy[c], static_cast<const RES *>(a.dy) + (size_t)row * a.ld_dy, c);
    }
  };
  Rows q;
  if (!WIDE && row_begin < row_end) fetch(q, row_begin);
  int par = 0, in_gate = 0;
  for (int row = row_begin, next; row < row_end; row = next, par ^= 1) {
    if (DIRECT) next = in_gate + 1 < a.rows_per_gate ? row + 1 : row + 1 + ((int)gridDim.x - 1) * a.rows_per_gate;
    else next = row + a.per_gate;
    Rows ahead;
    cols.fresh();
    if (WIDE) {
      q = Rows{};
      fetch(q, row);
    }
    if (!WIDE && next < row_end) fetch(ahead, next);
    float d[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) d[c][e] = 0.f;
    auto pre = [&](int c, int e) {  // u
      const float u = q.dh[c].at(e);
      return w_pre != nullptr ? u * w2[c].at(e) : u;
    };
    if (a.dh != nullptr) {
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        fence();
        if (!KEEP) load_pre(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float yn = q.y[c].at(e) * q.r2;
          s2.set(8 * c + e, __builtin_fmaf(q.dh[c].at(e), yn, s2.get(8 * c + e)));
          dot = __builtin_fmaf(pre(c, e), yn, dot);
        }
      }
      dot = row_sum(dot, slots[par][0]) * inv_d;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        q.y[c].forget();
        q.dh[c].forget();
        if (!KEEP) load_pre(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = q.r2 * (pre(c, e) - dot * (q.y[c].at(e) * q.r2));
      }
    }
    if (KEEP && DIRECT && in_gate == 0)
#pragma unroll
      for (int c = 0; c < NCH; ++c) load_gate(c);
    float dot = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      fence();
      if (!KEEP) {
        load_gate(c);
        load_post(c);
      }
      if (a.dy != nullptr)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = d[c][e] + q.dy[c].at(e);
      if (a.dx != nullptr) {
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = a.alpha * d[c][e];
        cols.template store<false>(static_cast<RES *>(a.dx) + (size_t)row * a.ld_dx, c, m);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float fn = q.f[c].at(e) * q.r1;
        s1.set(8 * c + e, __builtin_fmaf(d[c][e], fn, s1.get(8 * c + e)));
        d[c][e] = d[c][e] * gated(c, e) * post(c, e);
        dot = __builtin_fmaf(d[c][e], fn, dot);
      }
    }
    if (a.df != nullptr) {
      dot = a.post ? row_sum(dot, slots[par][1]) * inv_d : 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float m[8];
        q.f[c].forget();
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = q.r1 * (d[c][e] - dot * (q.f[c].at(e) * q.r1));
        cols.template store<false>(static_cast<ACT *>(a.df) + (size_t)row * a.ld_df, c, m);
      }
    }
    if (DIRECT && ++in_gate == a.rows_per_gate) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float m[8];
        if (!KEEP) {
          load_gate(c);
          load_post(c);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = s1.get(8 * c + e);
          m[e] = s * post(c, e);
          dw1.set(8 * c + e, __builtin_fmaf(gated(c, e), s, dw1.get(8 * c + e)));
          s1.set(8 * c + e, 0.f);
        }
        if (a.dgate != nullptr) cols.template store<false>(a.dgate + (size_t)gate_at * D, c, m);
      }
      in_gate = 0;
      gate_at += gridDim.x;
    }
    if (!WIDE) q = ahead;
  }
  const size_t mine = (size_t)blockIdx.x * D;
  const bool three = !DIRECT && a.part3 != nullptr;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    float m[8], n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = DIRECT ? dw1.get(8 * c + e) : s1.get(8 * c + e);
      n[e] = s2.get(8 * c + e);
    }
    cols.template store<false>(a.part2 + mine, c, n);
    if (three) {
      if (!KEEP) load_gate(c);
      cols.template store<false>(a.part3 + mine, c, m);
#pragma unroll
      for (int e = 0; e < 8; ++e) m[e] = m[e] * gated(c, e);
    }
    cols.template store<false>(a.part1 + mine, c, m);
  }
}

// The partial rows joined in a fixed order: 32 columns a workgroup, 32 threads a column, each
// adding every 32nd run.  y = 0: dw1 (with one gate or none the rows are S, which is dg's too);
// y = 1: dw2; y = 2 + g: gate g's dg.
template <class ACT>
__global__ __launch_bounds__(1024) void norm_gate_join_kernel(NormBwd a, int runs, bool one_gate) {
  __shared__ float part[32][33];
  const int c = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c, y = blockIdx.y;
  const bool in = col < a.D;
  const float *src = y == 0 ? a.part1 : y == 1 ? a.part2 : a.part3 + (size_t)(y - 2) * a.per_gate * a.D;
  const int n = y < 2 ? runs : a.per_gate;
  float s = 0.f;
  if (in) {
#pragma unroll 8
    for (int i = k; i < n; i += 32) s = s + src[(size_t)i * a.D + col];
  }
  part[k][c] = s;
  __syncthreads();
  if (k > 0 || !in) return;
  for (int i = 1; i < 32; ++i) s = s + part[i][c];
  if (y == 1) {
    if (a.dw_pre != nullptr) a.dw_pre[col] = s;
    return;
  }
  const float w1 = a.w_post != nullptr ? value(static_cast<const ACT *>(a.w_post)[col]) : 1.f;
  if (y >= 2) {
    a.dgate[(size_t)(y - 2) * a.D + col] = w1 * s;
    return;
  }
  if (one_gate) {
    if (a.dgate != nullptr) a.dgate[col] = w1 * s;
    if (a.gate != nullptr) s = s * value(static_cast<const ACT *>(a.gate)[col]);
  }
  if (a.dw_post != nullptr) a.dw_post[col] = s;
}

typedef void (*FwdFn)(NormFwd);
typedef void (*BwdFn)(NormBwd);

// Waves of a row at `per` chunks a thread, as threads.
int row_threads(int D, int per) { return std::min(1024, (chunks(D) + 64 * per - 1) / (64 * per) * 64); }
// The backward pass keeps up to 1024 chunks in registers.
bool wide_row(int D) { return D > 8192; }

template <bool REST, class ACT, class RES>
FwdFn fwd_fn(int nch) {
  return nch == 1 ? norm_gate_kernel<1, REST, ACT, RES> : norm_gate_kernel<2, REST, ACT, RES>;
}
template <class ACT, class RES>
int launch_fwd(const NormFwd &a, int num_cus, hipStream_t s) {
  // 16 columns a thread of a bf16 residual (8192 rows of 8192: 95 us, with 8 columns 112), 8 of a binary32 one
  // (20000 rows of 1505: 72 us, with 16 80); 8 too where rows are fewer than the CUs, for a row's way through its
  // two sums, and up to 512 columns, a wave's
  const bool one = sizeof(RES) == 4 || a.D <= 512 || a.rows <= num_cus;
  const int nch = one && a.D <= 8192 ? 1 : 2;
  const int rt = row_threads(a.D, nch);
  const FwdFn fn = a.D % 8 != 0 ? fwd_fn<true, ACT, RES>(nch) : fwd_fn<false, ACT, RES>(nch);
  // a grid's dimension counts at most 2^32 work-items: rows beyond 2^21 go on in the second one
  const int across = std::min(a.rows, 1 << 21);
  hipLaunchKernelGGL(fn, dim3(across, (a.rows + across - 1) / across), dim3(rt), 0, s, a);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

template <bool REST, class ACT, class RES>
BwdFn bwd_of(bool direct, bool wide) {
  return wide ? (direct ? norm_gate_bwd_kernel<2, REST, ACT, RES, true> : norm_gate_bwd_kernel<2, REST, ACT, RES, false>)
              : (direct ? norm_gate_bwd_kernel<1, REST, ACT, RES, true> : norm_gate_bwd_kernel<1, REST, ACT, RES, false>);
}
template <class ACT, class RES>
BwdFn bwd_fn(int D, bool direct, bool wide) {
  return D % 8 != 0 ? bwd_of<true, ACT, RES>(direct, wide) : bwd_of<false, ACT, RES>(direct, wide);
}

}  // namespace

// How a backward call is split.
NormSplit norm_split(int rows, int D, int groups) {
  NormSplit p{};
  p.rt = row_threads(D, wide_row(D) ? 2 : 1);
  if (rows == 0) return p;
  // at most one run a CU, or as many as make 512 threads: more fill the CUs no better, start unevenly and write
  // more partial rows (up to 1024 threads a CU: 16384 rows of 4096 bf16 165 us instead of 152,
  // 12004 of 5003 241 and 221, 32768 of 512 53 and 48).  Few rows make runs of up to 4.
  const int target = kNormRuns * std::max(1, 512 / p.rt);
  p.rows_per_gate = rows / groups;
  const int run = std::max((rows + target - 1) / target, std::min(4, (rows + kNormRuns - 1) / kNormRuns));
  p.direct = groups > 1 && p.rows_per_gate < run * 2;
  if (p.direct) {
    p.gates = std::max(1, run / p.rows_per_gate);
    p.runs = (groups + p.gates - 1) / p.gates;
  } else {
    p.run = std::min(run, p.rows_per_gate);
    p.per_gate = (p.rows_per_gate + p.run - 1) / p.run;
    p.runs = groups * p.per_gate;
  }
  return p;
}

size_t norm_bwd_workspace(int rows, int D, int groups) {
  const NormSplit p = norm_split(rows, D, groups);
  return (size_t)p.runs * D * sizeof(float) * (groups > 1 && !p.direct ? 3 : 2);
}

int norm_gate_launch(const occ_norm_args &n, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (n.rows == 0) return OCC_OK;
  NormFwd a{};
  a.rows = n.rows, a.D = n.D, a.post = n.post != 0, a.alpha = n.alpha, a.eps = n.eps;
  a.f = n.f, a.x = n.x, a.w_post = n.w_post, a.w_pre = n.w_pre, a.gate = n.gate;
  a.rows_per_gate = n.gate != nullptr ? n.rows / n.groups : 1;
  a.y = n.y, a.h = n.h, a.rstd = n.rstd;
  a.ld_f = n.ld_f, a.ld_x = n.ld_x, a.ld_y = n.ld_y, a.ld_h = n.ld_h;
  if (n.act == OCC_F32) return launch_fwd<float, float>(a, di->num_cus, s);
  return n.res == OCC_F32 ? launch_fwd<uint16_t, float>(a, di->num_cus, s) : launch_fwd<uint16_t, uint16_t>(a, di->num_cus, s);
}

int norm_gate_bwd_launch(const occ_norm_args &n, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  const int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  const int groups = n.gate != nullptr ? n.groups : 1;
  const NormSplit p = norm_split(n.rows, n.D, groups);
  NormBwd a{};
  a.rows = n.rows, a.D = n.D, a.post = n.post != 0, a.alpha = n.alpha;
  a.f = n.f, a.y = n.y, a.dy = n.dy, a.dh = n.dh, a.w_post = n.w_post, a.w_pre = n.w_pre, a.gate = n.gate;
  a.rstd = n.rstd, a.df = n.df, a.dx = n.dx, a.dw_post = n.dw_post, a.dw_pre = n.dw_pre, a.dgate = n.dgate;
  a.ld_f = n.ld_f, a.ld_y = n.ld_y, a.ld_dy = n.ld_dy, a.ld_dh = n.ld_dh, a.ld_df = n.ld_df, a.ld_dx = n.ld_dx;
  a.rows_per_gate = p.rows_per_gate, a.per_gate = p.per_gate;
  a.part1 = static_cast<float *>(n.workspace);
  a.part2 = a.part1 + (size_t)p.runs * n.D;
  const bool three = groups > 1 && !p.direct;
  a.part3 = three ? a.part2 + (size_t)p.runs * n.D : nullptr;
  if (n.rows > 0) {
    const bool wide = wide_row(n.D);
    const int lds = wide ? 2 * 16 * 1024 * (int)sizeof(float) : 0;
    BwdFn fn;
    if (n.act == OCC_F32) fn = bwd_fn<float, float>(n.D, p.direct, wide);
    else if (n.res == OCC_F32) fn = bwd_fn<uint16_t, float>(n.D, p.direct, wide);
    else fn = bwd_fn<uint16_t, uint16_t>(n.D, p.direct, wide);
    if (wide && hipFuncSetAttribute(reinterpret_cast<const void *>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
      return OCC_EHIP;
    hipLaunchKernelGGL(fn, dim3(p.runs), dim3(p.rt), lds, s, a);
    if (hipGetLastError() != hipSuccess) return OCC_EHIP;
  }
  // without rows the sums are empty and the join writes their zeros
  const bool gates = three && n.dgate != nullptr;
  hipLaunchKernelGGL(n.act == OCC_F32 ? norm_gate_join_kernel<float> : norm_gate_join_kernel<uint16_t>,
                     dim3((n.D + 31) / 32, gates ? 2 + groups : 2), dim3(1024), 0, s, a, p.runs, groups == 1);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace occ
