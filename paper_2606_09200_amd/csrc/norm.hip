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
// parameters are binary32; rows are rounded once, when stored (h from the unrounded y).
#include "block_util.h"

#include <algorithm>

namespace occ {
namespace {

// Sum over the RT threads of a row; `slot` holds RT / 64 floats that no one else uses
// before the next barrier but one.  The order of the sum is fixed.
template <int RT>
__device__ __forceinline__ float row_sum(float v, float *slot) {
  v = wave_sum(v);
  if constexpr (RT > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) slot[wave] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int w = 1; w < RT / 64; ++w) v = v + slot[w];
  }
  return v;
}

// ---------------------------------------------------------------------------
// Forward.  RT threads to a row, NCH chunks of 8 columns a thread (chunk c of thread
// t: columns 8 (c RT + t)); a workgroup of max(RT, 256) threads walks rows with the
// grid's stride.  One wave per row needs no barrier.
template <int RT, int NCH, class ACT, class RES>
__global__ __launch_bounds__(RT > 256 ? RT : 256) void norm_gate_kernel(NormFwd a) {
  constexpr int NT = RT > 256 ? RT : 256, RPW = NT / RT;
  __shared__ float slots[2][2][16];
  const int t = threadIdx.x % RT;
  const ACT *w1 = static_cast<const ACT *>(a.w_post), *w2 = static_cast<const ACT *>(a.w_pre);
  const float inv_d = 1.0f / (float)a.D;
  int par = 0;
  for (int row0 = blockIdx.x * RPW; row0 < a.rows; row0 += gridDim.x * RPW, par ^= 1) {
    const int row = row0 + (RPW > 1 ? threadIdx.x / RT : 0);
    const bool live = RPW == 1 || row < a.rows;
    const int D = live ? a.D : 0;
    const ACT *f = static_cast<const ACT *>(a.f) + (live ? (size_t)row * a.ld_f : 0);
    const RES *x = static_cast<const RES *>(a.x) + (live ? (size_t)row * a.ld_x : 0);
    const ACT *gate = static_cast<const ACT *>(a.gate);
    if (gate != nullptr && live) gate += (size_t)(row / a.rows_per_gate) * a.D;
    float fv[NCH][8], yv[NCH][8];
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * RT + t) * 8;
      load8(f + min(at, D), D - at, fv[c]);
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * RT + t) * 8;
      load8(x + min(at, D), D - at, yv[c]);
    }
    float r1 = 1.f;
    if (a.post) {
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(fv[c][e], fv[c][e], ss);
      r1 = 1.0f / __builtin_sqrtf(row_sum<RT>(ss, slots[par][0]) * inv_d + a.eps);
    }
    ss = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int at = (c * RT + t) * 8;
      float m[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) m[e] = fv[c][e] * r1;
      if (w1 != nullptr) {
        float w[8];
        load8(w1 + min(at, D), D - at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = m[e] * w[e];
      }
      if (gate != nullptr) {
        float w[8];
        load8(gate + min(at, D), D - at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = m[e] * w[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        yv[c][e] = __builtin_fmaf(a.alpha, yv[c][e], m[e]);
        ss = __builtin_fmaf(yv[c][e], yv[c][e], ss);
      }
      store8(static_cast<RES *>(a.y) + (size_t)row * a.ld_y + at, D - at, yv[c]);
    }
    float r2 = 1.f;
    if (a.h != nullptr) {
      r2 = 1.0f / __builtin_sqrtf(row_sum<RT>(ss, slots[par][1]) * inv_d + a.eps);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int at = (c * RT + t) * 8;
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = yv[c][e] * r2;
        if (w2 != nullptr) {
          float w[8];
          load8(w2 + min(at, D), D - at, w);
#pragma unroll
          for (int e = 0; e < 8; ++e) m[e] = m[e] * w[e];
        }
        store8(static_cast<ACT *>(a.h) + (size_t)row * a.ld_h + at, D - at, m);
      }
    }
    if (a.rstd != nullptr && t == 0 && live) {
      a.rstd[2 * (size_t)row] = r1;
      a.rstd[2 * (size_t)row + 1] = r2;
    }
  }
}

// ---------------------------------------------------------------------------
// Backward.  A workgroup of RT threads takes a run of rows, NCH chunks of 8 columns a
// thread, and keeps the sums over its rows; the next row's loads are in flight
// while a row is worked on.
//
// Where gates are shared by many rows (or there is none), a run stays within one
// gate's rows (`per_gate` runs each).  S and dw2's sum leave as one row each of the
// partial arrays; with several gates g S does too, as the first.  Where gates are not
// shared so (DIRECT), a run is `gates` whole gates: at the end of each, dg is
// complete and stored, and g S goes into the run's sum of dw1, the first array's row.
//
// Up to 8192 columns (NCH = 1) the sums, the weights and two rows fit in registers.
// Beyond (NCH = 2, 1024 threads of 128 registers) the sums live in LDS, the
// weights come from the caches for each row, and rows are not fetched ahead.
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
  float *at;  // this thread's words, blockDim.x apart: no bank conflicts, no barriers
  __device__ __forceinline__ explicit ColumnSums(float *base) : at(base + threadIdx.x) {
#pragma unroll
    for (int i = 0; i < N; ++i) set(i, 0.f);
  }
  __device__ __forceinline__ float get(int i) const { return at[i * 1024]; }
  __device__ __forceinline__ void set(int i, float x) { at[i * 1024] = x; }
};

template <int RT, int NCH, class ACT, class RES, bool DIRECT>
__global__ __launch_bounds__(RT) void norm_gate_bwd_kernel(NormBwd a) {
  constexpr bool WIDE = NCH > 1;
  static_assert(!WIDE || RT == 1024, "ColumnSums' stride");
  __shared__ float slots[2][2][16];
  extern __shared__ __align__(16) unsigned char smem[];  // WIDE: two arrays of 8 NCH RT sums
  float *lds = reinterpret_cast<float *>(smem);
  const int D = a.D;
  const float inv_d = 1.0f / (float)D;
  int row_begin, row_end, gate_at;
  if (DIRECT) {
    gate_at = blockIdx.x * a.gates;
    row_begin = gate_at * a.rows_per_gate;
    row_end = min(a.rows, row_begin + a.gates * a.rows_per_gate);
  } else {
    gate_at = blockIdx.x / a.per_gate;
    row_begin = gate_at * a.rows_per_gate + (int)(blockIdx.x % a.per_gate) * a.run;
    row_end = min((gate_at + 1) * a.rows_per_gate, row_begin + a.run);
  }
  uint32_t at[NCH];  // first column of a chunk
  int left[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    at[c] = (uint32_t)(c * RT + (int)threadIdx.x) * 8u;
    left[c] = D - (int)at[c];
  }
  const ACT *w_post = static_cast<const ACT *>(a.w_post), *w_pre = static_cast<const ACT *>(a.w_pre);
  const ACT *gate = static_cast<const ACT *>(a.gate);
  Raw8<ACT> w1[NCH], w2[NCH], gv[NCH];
  auto load_gate = [&]() {
    if (gate != nullptr)
#pragma unroll
      for (int c = 0; c < NCH; ++c) gv[c].load(element(gate + (size_t)gate_at * D, at[c]), left[c]);
  };
  auto load_post = [&]() {
    if (w_post != nullptr)
#pragma unroll
      for (int c = 0; c < NCH; ++c) w1[c].load(element(w_post, at[c]), left[c]);
  };
  auto load_pre = [&]() {
    if (w_pre != nullptr)
#pragma unroll
      for (int c = 0; c < NCH; ++c) w2[c].load(element(w_pre, at[c]), left[c]);
  };
  auto post = [&](int c, int e) { return w_post != nullptr ? w1[c].at(e) : 1.f; };
  auto gated = [&](int c, int e) { return gate != nullptr ? gv[c].at(e) : 1.f; };
  // S: of the run, or (DIRECT) of the gate; dw1: DIRECT only
  ColumnSums<8 * NCH, WIDE && !DIRECT> s1(lds);
  ColumnSums<8 * NCH, WIDE> s2(lds + 8 * NCH * RT);
  ColumnSums<8 * NCH, WIDE && DIRECT> dw1(lds);
  if (!WIDE) {
    load_post();
    load_pre();
    if (!DIRECT) load_gate();
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
        q.y[c].load(element(static_cast<const RES *>(a.y) + (size_t)row * a.ld_y, at[c]), left[c]);
        q.dh[c].load(element(static_cast<const ACT *>(a.dh) + (size_t)row * a.ld_dh, at[c]), left[c]);
      }
      q.f[c].load(element(static_cast<const ACT *>(a.f) + (size_t)row * a.ld_f, at[c]), left[c]);
      if (a.dy != nullptr) q.dy[c].load(element(static_cast<const RES *>(a.dy) + (size_t)row * a.ld_dy, at[c]), left[c]);
    }
  };
  Rows q;
  if (!WIDE && row_begin < row_end) fetch(q, row_begin);
  int par = 0, in_gate = 0;
  for (int row = row_begin; row < row_end; ++row, par ^= 1) {
    Rows ahead;
    if (WIDE) fetch(q, row);
    else fetch(ahead, min(row + 1, row_end - 1));
    float d[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) d[c][e] = 0.f;
    if (a.dh != nullptr) {
      if (WIDE) load_pre();
      float yn[NCH][8], u[NCH][8];
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          yn[c][e] = q.y[c].at(e) * q.r2;
          u[c][e] = q.dh[c].at(e);
          s2.set(8 * c + e, __builtin_fmaf(u[c][e], yn[c][e], s2.get(8 * c + e)));
          if (w_pre != nullptr) u[c][e] = u[c][e] * w2[c].at(e);
          dot = __builtin_fmaf(u[c][e], yn[c][e], dot);
        }
      dot = row_sum<RT>(dot, slots[par][0]) * inv_d;
#pragma unroll
      for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = q.r2 * (u[c][e] - dot * yn[c][e]);
    }
    if (WIDE) load_post();
    if (DIRECT ? WIDE || in_gate == 0 : WIDE) load_gate();
    float dot = 0.f;
    float fn[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      if (a.dy != nullptr)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[c][e] = d[c][e] + q.dy[c].at(e);
      if (a.dx != nullptr) {
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = a.alpha * d[c][e];
        store8(element(static_cast<RES *>(a.dx) + (size_t)row * a.ld_dx, at[c]), left[c], m);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        fn[c][e] = q.f[c].at(e) * q.r1;
        s1.set(8 * c + e, __builtin_fmaf(d[c][e], fn[c][e], s1.get(8 * c + e)));
        d[c][e] = d[c][e] * gated(c, e) * post(c, e);
        dot = __builtin_fmaf(d[c][e], fn[c][e], dot);
      }
    }
    if (a.df != nullptr) {
      dot = a.post ? row_sum<RT>(dot, slots[par][1]) * inv_d : 0.f;
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = q.r1 * (d[c][e] - dot * fn[c][e]);
        store8(element(static_cast<ACT *>(a.df) + (size_t)row * a.ld_df, at[c]), left[c], m);
      }
    }
    if (DIRECT && ++in_gate == a.rows_per_gate) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = s1.get(8 * c + e);
          m[e] = s * post(c, e);
          dw1.set(8 * c + e, __builtin_fmaf(gated(c, e), s, dw1.get(8 * c + e)));
          s1.set(8 * c + e, 0.f);
        }
        if (a.dgate != nullptr) store8(element(a.dgate + (size_t)gate_at * D, at[c]), left[c], m);
      }
      in_gate = 0;
      ++gate_at;
    }
    if (!WIDE) q = ahead;
  }
  const size_t mine = (size_t)blockIdx.x * D;
  const bool three = !DIRECT && a.part3 != nullptr;
  if (WIDE && three) load_gate();
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    float m[8], n[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = DIRECT ? dw1.get(8 * c + e) : s1.get(8 * c + e);
      n[e] = s2.get(8 * c + e);
    }
    store8(element(a.part2 + mine, at[c]), left[c], n);
    if (three) {
      store8(element(a.part3 + mine, at[c]), left[c], m);
#pragma unroll
      for (int e = 0; e < 8; ++e) m[e] = m[e] * gated(c, e);
    }
    store8(element(a.part1 + mine, at[c]), left[c], m);
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
  if (in)
    for (int i = k; i < n; i += 32) s = s + src[(size_t)i * a.D + col];
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

// Threads per row and chunks per thread by width; with few rows, more threads a row shorten a
// row's way through its two sums.
template <class ACT, class RES>
int launch_fwd(const NormFwd &a, int num_cus, hipStream_t s) {
  const bool few = a.rows <= num_cus;
  FwdFn fn;
  int rt;
  if (a.D <= 512) fn = norm_gate_kernel<64, 1, ACT, RES>, rt = 64;
  else if (a.D <= 1024 && !few) fn = norm_gate_kernel<64, 2, ACT, RES>, rt = 64;
  else if (a.D <= 2048) fn = norm_gate_kernel<256, 1, ACT, RES>, rt = 256;
  else if (few && a.D <= 8192) fn = norm_gate_kernel<1024, 1, ACT, RES>, rt = 1024;
  else if (few) fn = norm_gate_kernel<1024, 2, ACT, RES>, rt = 1024;
  else if (a.D <= 4096) fn = norm_gate_kernel<256, 2, ACT, RES>, rt = 256;
  else if (a.D <= 8192) fn = norm_gate_kernel<256, 4, ACT, RES>, rt = 256;
  else fn = norm_gate_kernel<256, 8, ACT, RES>, rt = 256;
  const int nt = rt > 256 ? rt : 256, rpw = nt / rt;
  const int grid = std::min((a.rows + rpw - 1) / rpw, num_cus * 8);
  hipLaunchKernelGGL(fn, dim3(grid), dim3(nt), 0, s, a);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

template <class ACT, class RES, bool DIRECT>
BwdFn bwd_fn(int rt, bool wide) {
  return wide ? norm_gate_bwd_kernel<1024, 2, ACT, RES, DIRECT>
       : rt == 64 ? norm_gate_bwd_kernel<64, 1, ACT, RES, DIRECT> : rt == 128 ? norm_gate_bwd_kernel<128, 1, ACT, RES, DIRECT>
       : rt == 256 ? norm_gate_bwd_kernel<256, 1, ACT, RES, DIRECT> : rt == 512 ? norm_gate_bwd_kernel<512, 1, ACT, RES, DIRECT>
                   : norm_gate_bwd_kernel<1024, 1, ACT, RES, DIRECT>;
}

}  // namespace

// How a backward call is split.
NormSplit norm_split(int rows, int D, int groups) {
  NormSplit p{};
  p.rt = 64;
  while (p.rt < 1024 && p.rt * 8 < D) p.rt *= 2;
  if (rows == 0) return p;
  // at most kNormRuns * 1024 / rt runs: a workgroup of 1024 threads per CU or its equal in
  // threads; more would write more partial rows than they gain in load balance
  const int target = kNormRuns * 1024 / p.rt;
  p.rows_per_gate = rows / groups;
  const int run = (rows + target - 1) / target;
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
  a.rows_per_gate = p.rows_per_gate, a.run = p.run, a.per_gate = p.per_gate, a.gates = p.gates;
  a.part1 = static_cast<float *>(n.workspace);
  a.part2 = a.part1 + (size_t)p.runs * n.D;
  const bool three = groups > 1 && !p.direct;
  a.part3 = three ? a.part2 + (size_t)p.runs * n.D : nullptr;
  if (n.rows > 0) {
    const bool wide = n.D > 8192;
    const int lds = wide ? 2 * 16 * 1024 * (int)sizeof(float) : 0;
    BwdFn fn;
    if (n.act == OCC_F32) fn = p.direct ? bwd_fn<float, float, true>(p.rt, wide) : bwd_fn<float, float, false>(p.rt, wide);
    else if (n.res == OCC_F32) fn = p.direct ? bwd_fn<uint16_t, float, true>(p.rt, wide) : bwd_fn<uint16_t, float, false>(p.rt, wide);
    else fn = p.direct ? bwd_fn<uint16_t, uint16_t, true>(p.rt, wide) : bwd_fn<uint16_t, uint16_t, false>(p.rt, wide);
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
