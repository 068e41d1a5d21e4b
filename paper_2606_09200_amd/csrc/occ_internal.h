// Internal interfaces of the occ library (not part of the public ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/occ.h"
#include "device_util.h"

namespace occ {

constexpr int kMaxReduceChunks = 64;
constexpr int kMaxPermuteChunks = 512;

// Per-device facts the launch plans depend on (queried once per device).
struct DeviceInfo {
  int ok;
  int num_cus;
  int lds_per_cu;       // bytes
  int max_lds_per_wg;   // bytes
  int clock_khz;
  int gfx950;
};
const DeviceInfo &device_info(int device);
int current_device_info(const DeviceInfo **out);

// ---- GEMM ----------------------------------------------------------------
struct GemmCall {
  const void *A;
  const void *B;
  void *C;
  int M, N, K;
  size_t lds_bytes;
  int grid_cap;         // 0 = one workgroup per tile
  int variant;          // 0 = automatic, else a kernel variant id
  int priority;         // wave priority 0..3 (s_setprio)
  KHooks trace;         // per-launch hooks: tracing, dependency counter (all off by default)
  bool b_kn = false;    // B stored K x N (occ_gemm: C = A B) or N x K (occ_gemm_bt: C = A B^T)
};
int gemm_plan(const GemmCall &c, occ_gemm_plan *plan);
// the plan without the occupancy figure (wg_per_cu = 0): no runtime query
int gemm_launch_plan(const GemmCall &c, occ_gemm_plan *plan);
bool gemm_variant_is_kn(int id);  // a variant that takes B stored K x N
int gemm_launch(const GemmCall &c, hipStream_t s);

// ---- communication-side kernels -----------------------------------------
struct ReduceCall {
  const float *const *bufs;  // host array
  int nchunks;
  size_t len;
  float *out;
  int wgs;                   // 0 = default
  int priority;              // 0..3
  KHooks trace;
  double rate_gbs;           // target bandwidth of the vector path, GB/s; 0 = unpaced
  // when set: the first term of every sum is this bf16 buffer, widened to
  // binary32, and bufs holds the nchunks (>= 0) fp32 terms after it
  const uint16_t *own = nullptr;
};
int reduce_launch(const ReduceCall &c, hipStream_t s);
int reduce_default_wgs(const ReduceCall &c);

struct PermuteCall {
  const void *src;
  void *dst;
  const int32_t *perm;       // host array
  int nchunks;
  size_t chunk_bytes;
  int wgs;
  int priority;
  KHooks trace;
  double rate_gbs;           // as ReduceCall::rate_gbs
};
int permute_launch(const PermuteCall &c, hipStream_t s);
int permute_default_wgs(const PermuteCall &c);

// ---- validation (host only, no HIP calls) --------------------------------
int validate_gemm(const void *A, const void *B, const void *C, int M, int N, int K, bool b_kn = false);
int validate_reduce(const float *const *bufs, int nchunks, size_t len, const float *out);
int validate_reduce_own(const void *own, const float *const *peers, int npeers, size_t len, const float *out);
int validate_permute(const void *src, const void *dst, const int32_t *perm, int nchunks,
                     size_t chunk_bytes);

// ---- operators of a block (include/occ.h) ---------------------------------
struct Mx4QuantCall {
  const void *x;
  int dtype, rows, cols;
  size_t ld;
  void *codes, *scales;      // of x, or null
  void *codes_t, *scales_t;  // of its transpose, or null
};
int validate_mx4_quant(const Mx4QuantCall &c);
int mx4_quant_launch(const Mx4QuantCall &c, hipStream_t s);

struct Mx4DequantCall {
  const void *codes, *scales;
  int rows, cols;
  void *out;
  int dtype;
  size_t ld;
};
int validate_mx4_dequant(const Mx4DequantCall &c);
int mx4_dequant_launch(const Mx4DequantCall &c, hipStream_t s);

struct Mx4GemmCall {
  const void *A, *As, *B, *Bs;
  void *C;
  int dtype, M, N, K;
  size_t lds_bytes;
};
int validate_mx4_gemm_dims(int M, int N, int K);
int validate_mx4_gemm(const Mx4GemmCall &c);
int mx4_gemm_launch(const Mx4GemmCall &c, hipStream_t s);
void mx4_gemm_plan(int M, int N, int K, int num_cus, occ_gemm_mx4_plan *plan);

struct NormFwd {
  int rows, D;
  bool post;
  float alpha, eps;
  const void *f, *x, *w_post, *w_pre, *gate;
  int rows_per_gate;
  void *y, *h;
  float *rstd;
  size_t ld_f, ld_x, ld_y, ld_h;
};
struct NormBwd {
  int rows, D;
  bool post;
  float alpha;
  const void *f, *y, *dy, *dh, *w_post, *w_pre, *gate;
  const float *rstd;
  void *df, *dx;
  float *dw_post, *dw_pre, *dgate;
  size_t ld_f, ld_y, ld_dy, ld_dh, ld_df, ld_dx;
  int rows_per_gate, per_gate;  // see NormSplit
  float *part1, *part2, *part3;  // runs x D each; part3 only where several gates have several runs
};
// The backward's runs of rows: either `per_gate` runs of at most `run` rows within each gate's
// rows, or (direct) runs of up to `gates` whole gates.  rt: threads a run.
struct NormSplit {
  int rt, runs, rows_per_gate;
  bool direct;
  int run, per_gate, gates;
};
constexpr int kNormRuns = 256;
NormSplit norm_split(int rows, int D, int groups);
size_t norm_bwd_workspace(int rows, int D, int groups);
int validate_norm(const occ_norm_args &n, bool backward);
int norm_gate_launch(const occ_norm_args &n, hipStream_t s);
int norm_gate_bwd_launch(const occ_norm_args &n, hipStream_t s);

struct MoeCounters {
  uint32_t arrived;  // router workgroups that are done; zero between calls
  uint32_t active;   // experts that some token picked
};
struct MoeExpert {
  uint32_t id, first, n;  // its index, its first row of the hidden activations, their number
  uint32_t unused;
};
struct MoeRow {  // of the hidden activations: a token's with one of its experts
  int token;
  float weight;
};
struct MoeMatrix {
  const void *w;
  const uint8_t *scales;
  size_t stride, scale_stride;  // bytes from expert to expert
};
struct MoeCall {
  int T, H, I, E, k;
  bool renorm;
  int slices, row_blocks, max_segments, ld_x, rbs;
  const uint16_t *x, *router;
  MoeMatrix gate, up, down;
  const uint8_t *mask;
  uint16_t *y;
  size_t ld_y;
  int32_t *ids;
  float *weights;
  // workspace
  MoeCounters *count;
  MoeExpert *plan;
  MoeRow *rows;
  uint32_t *joined;  // per 32 rows of y: finished parts
  float *part;       // partial logits
  uint16_t *hidden;  // rows x 2 x I, bf16: the upper and lower halves
  float *sums;       // parts x T x H
};
int validate_moe_sizes(int T, int H, int I, int E, int k);
int validate_moe(const occ_moe_args &a);
size_t moe_workspace(int T, int H, int I, int E, int k);
int moe_launch(const occ_moe_args &a, hipStream_t s);

int validate_kv_tables(const occ_kv_tables_args &a);
int kv_tables_launch(const occ_kv_tables_args &a, hipStream_t s);
int validate_rope(const occ_rope_args &a);
int rope_launch(const occ_rope_args &a, hipStream_t s);
bool attn_heads(int Hq, int Hkv, int D);
int validate_attn(const occ_attn_args &a);
size_t attn_workspace(int D);
int attn_launch(const occ_attn_args &a, hipStream_t s);

// Tracing helper: sets npairs [start, end] pairs to [UINT64_MAX, 0] and the
// workgroup-record counter wg[0] to 0 (either pointer may be null).
int trace_reset(uint64_t *stamps, int npairs, uint32_t *wg, hipStream_t s);

}  // namespace occ
