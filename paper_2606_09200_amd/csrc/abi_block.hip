// Public C entry points of the operators of a block: argument validation (host
// only, before any HIP call) and dispatch.
#include "occ_internal.h"

namespace occ {
namespace {

bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

struct Range {
  const void *p;
  size_t bytes;
};

bool overlaps(const Range &a, const Range &b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// No output overlaps an input or another output.
template <int NO, int NI>
bool disjoint(const Range (&out)[NO], const Range (&in)[NI]) {
  for (int i = 0; i < NO; ++i) {
    for (int j = 0; j < NI; ++j)
      if (overlaps(out[i], in[j])) return false;
    for (int j = 0; j < i; ++j)
      if (overlaps(out[i], out[j])) return false;
  }
  return true;
}

bool float_type(int dtype) { return dtype == OCC_BF16 || dtype == OCC_F32; }
size_t type_bytes(int dtype) { return dtype == OCC_F32 ? 4 : 2; }

// Bytes a rows x cols matrix with row pitch ld spans.
size_t span(int rows, int cols, size_t ld, int dtype) {
  return rows == 0 || cols == 0 ? 0 : ((size_t)(rows - 1) * ld + cols) * type_bytes(dtype);
}

bool mx4_dims(int rows, int cols) {
  return rows >= 0 && cols >= 0 && rows <= OCC_MX4_MAX_DIM && cols <= OCC_MX4_MAX_DIM;
}

bool mx4_pointers(const void *codes, const void *scales) {
  return codes != nullptr && scales != nullptr && aligned(codes, 16) && aligned(scales, 16);
}

}  // namespace

int validate_mx4_quant(const Mx4QuantCall &c) {
  if (!float_type(c.dtype) || !mx4_dims(c.rows, c.cols) || c.ld < (size_t)c.cols) return OCC_EINVAL;
  if ((c.codes == nullptr) != (c.scales == nullptr) || (c.codes_t == nullptr) != (c.scales_t == nullptr)) return OCC_EINVAL;
  if (c.codes == nullptr && c.codes_t == nullptr) return OCC_EINVAL;
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  // a grid counts at most 2^32 work-items: 2^24 - 1 workgroups of 256
  const unsigned long long wgs = c.codes_t == nullptr
                                     ? ((c.rows + 15ull) / 16) * ((c.cols + 511ull) / 512)
                                     : ((c.rows + 511ull) / 512 * 4) * ((c.cols + 511ull) / 512 * 4);
  if (wgs >= (1ull << 24)) return OCC_EINVAL;
  if (c.x == nullptr || !aligned(c.x, type_bytes(c.dtype))) return OCC_EINVAL;
  if (c.codes != nullptr && !mx4_pointers(c.codes, c.scales)) return OCC_EINVAL;
  if (c.codes_t != nullptr && !mx4_pointers(c.codes_t, c.scales_t)) return OCC_EINVAL;
  const Range in[] = {{c.x, span(c.rows, c.cols, c.ld, c.dtype)}};
  const Range out[] = {{c.codes, OCC_MX4_CODE_BYTES(c.rows, c.cols)}, {c.scales, OCC_MX4_SCALE_BYTES(c.rows, c.cols)},
                       {c.codes_t, OCC_MX4_CODE_BYTES(c.cols, c.rows)},
                       {c.scales_t, OCC_MX4_SCALE_BYTES(c.cols, c.rows)}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

int validate_mx4_dequant(const Mx4DequantCall &c) {
  if (!float_type(c.dtype) || !mx4_dims(c.rows, c.cols) || c.ld < (size_t)c.cols) return OCC_EINVAL;
  if (c.rows == 0 || c.cols == 0) return OCC_OK;
  if (!mx4_pointers(c.codes, c.scales) || c.out == nullptr || !aligned(c.out, type_bytes(c.dtype))) return OCC_EINVAL;
  const Range in[] = {{c.codes, OCC_MX4_CODE_BYTES(c.rows, c.cols)}, {c.scales, OCC_MX4_SCALE_BYTES(c.rows, c.cols)}};
  const Range out[] = {{c.out, span(c.rows, c.cols, c.ld, c.dtype)}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

int validate_mx4_gemm_dims(int M, int N, int K) {
  if (!mx4_dims(M, N) || !mx4_dims(M, K)) return OCC_EINVAL;
  // the grid of the smallest tile (32 x 64) in work-items, as above
  return ((M + 31ull) / 32) * ((N + 63ull) / 64) >= (1ull << 23) ? OCC_EINVAL : OCC_OK;
}

int validate_mx4_gemm(const Mx4GemmCall &c) {
  if (!float_type(c.dtype) || validate_mx4_gemm_dims(c.M, c.N, c.K) != OCC_OK) return OCC_EINVAL;
  if (c.M == 0 || c.N == 0) return OCC_OK;
  if (c.C == nullptr || !aligned(c.C, type_bytes(c.dtype))) return OCC_EINVAL;
  if (c.K > 0 && (!mx4_pointers(c.A, c.As) || !mx4_pointers(c.B, c.Bs))) return OCC_EINVAL;
  const Range in[] = {{c.A, OCC_MX4_CODE_BYTES(c.M, c.K)}, {c.As, OCC_MX4_SCALE_BYTES(c.M, c.K)},
                      {c.B, OCC_MX4_CODE_BYTES(c.N, c.K)}, {c.Bs, OCC_MX4_SCALE_BYTES(c.N, c.K)}};
  const Range out[] = {{c.C, span(c.M, c.N, c.N, c.dtype)}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

namespace {

// out may also be exactly one of the inputs (same pitch): in place, row by row.
bool in_place(const Range &out, const Range &in, size_t ld_out, size_t ld_in) {
  return out.p != nullptr && out.p == in.p && ld_out == ld_in;
}

}  // namespace

int validate_norm(const occ_norm_args &n, bool backward) {
  if (!float_type(n.act) || !float_type(n.res) || (n.act == OCC_F32 && n.res != OCC_F32)) return OCC_EINVAL;
  if (n.rows < 0 || n.rows > (1 << 30) || n.D < 1 || n.D > OCC_NORM_MAX_D) return OCC_EINVAL;
  if (n.post == 0 && (n.w_post != nullptr || (backward && n.dw_post != nullptr))) return OCC_EINVAL;
  if (n.gate != nullptr &&
      (n.groups < 1 || (n.rows > 0 ? n.groups > n.rows || n.rows % n.groups != 0 : n.groups > 65533)))
    return OCC_EINVAL;
  if (backward && n.gate == nullptr && n.dgate != nullptr) return OCC_EINVAL;
  const size_t ea = type_bytes(n.act), er = type_bytes(n.res), D = (size_t)n.D;
  const size_t gates = n.gate != nullptr ? (size_t)n.groups * D * ea : 0;
  if (!aligned(n.w_post, ea) || !aligned(n.w_pre, ea) || !aligned(n.gate, ea)) return OCC_EINVAL;
  struct Rows {
    const void *p;
    size_t ld, elem;
    bool needed;
  };
  auto bad = [&](const Rows &r) {
    return n.rows > 0 && ((r.needed && r.p == nullptr) || (r.p != nullptr && (!aligned(r.p, r.elem) || r.ld < D)));
  };
  auto range = [&](const Rows &r) {
    return Range{r.p, n.rows == 0 ? 0 : ((size_t)(n.rows - 1) * r.ld + D) * r.elem};
  };
  const Rows f{n.f, n.ld_f, ea, true}, y{n.y, n.ld_y, er, !backward || n.dh != nullptr};
  const Range wp{n.w_post, D * ea}, wq{n.w_pre, D * ea}, g{n.gate, gates};
  const Range rstd{n.rstd, (size_t)n.rows * 8};
  if (!aligned(n.rstd, 4) || bad(f) || bad(y)) return OCC_EINVAL;
  if (!backward) {
    const Rows x{n.x, n.ld_x, er, true}, h{n.h, n.ld_h, ea, false};
    if (bad(x) || bad(h)) return OCC_EINVAL;
    const Range none{nullptr, 0};
    const Range in[] = {in_place(range(h), range(f), h.ld, f.ld) ? none : range(f),
                        in_place(range(y), range(x), y.ld, x.ld) ? none : range(x), wp, wq, g};
    const Range out[] = {range(y), range(h), rstd};
    // in place or not, y stays off f and h off x
    if (overlaps(range(y), range(f)) || overlaps(range(h), range(x))) return OCC_EALIAS;
    return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
  }
  const Rows dy{n.dy, n.ld_dy, er, false}, dh{n.dh, n.ld_dh, ea, false};
  const Rows df{n.df, n.ld_df, ea, false}, dx{n.dx, n.ld_dx, er, false};
  if (n.rows > 0 && ((n.dy == nullptr && n.dh == nullptr) || n.rstd == nullptr)) return OCC_EINVAL;
  if (bad(dy) || bad(dh) || bad(df) || bad(dx)) return OCC_EINVAL;
  if (!aligned(n.dw_post, 4) || !aligned(n.dw_pre, 4) || !aligned(n.dgate, 4)) return OCC_EINVAL;
  const size_t need = norm_bwd_workspace(n.rows, n.D, n.gate != nullptr ? n.groups : 1);
  if (need > 0 && (n.workspace == nullptr || !aligned(n.workspace, 16) || n.workspace_bytes < need)) return OCC_EINVAL;
  const Range out[] = {range(df), range(dx), {n.dw_post, D * 4}, {n.dw_pre, D * 4},
                       {n.dgate, n.gate != nullptr ? (size_t)n.groups * D * 4 : 0}, {n.workspace, need}};
  const Range none{nullptr, 0};
  const Range rest[] = {range(y), wp, wq, g, rstd, none};
  if (!disjoint(out, rest)) return OCC_EALIAS;
  for (const Range &o : out) {
    if (overlaps(o, range(f)) && !(o.p == n.df && in_place(o, range(f), n.ld_df, n.ld_f))) return OCC_EALIAS;
    if (overlaps(o, range(dh)) && !(o.p == n.df && in_place(o, range(dh), n.ld_df, n.ld_dh))) return OCC_EALIAS;
    if (overlaps(o, range(dy)) && !(o.p == n.dx && in_place(o, range(dy), n.ld_dx, n.ld_dy))) return OCC_EALIAS;
  }
  return OCC_OK;
}

int validate_moe(const occ_moe_args &a) {
  const int st = validate_moe_sizes(a.tokens, a.H, a.I, a.experts, a.top_k);
  if (st != OCC_OK) return st;
  const bool mx = a.weight_type == OCC_MX4;
  if (!mx && a.weight_type != OCC_BF16) return OCC_EINVAL;
  if (a.tokens == 0) return OCC_OK;
  const size_t H = (size_t)a.H, I = (size_t)a.I, E = (size_t)a.experts, T = (size_t)a.tokens, k = (size_t)a.top_k;
  if (a.x == nullptr || a.router == nullptr || a.y == nullptr || !aligned(a.x, 16) || !aligned(a.router, 16) ||
      !aligned(a.y, 2) || !aligned(a.ids, 4) || !aligned(a.weights, 4))
    return OCC_EINVAL;
  // rows of x are addressed with 32-bit byte offsets
  if (a.ld_x < H || a.ld_x % 8 != 0 || a.ld_x > (1u << 23) || a.ld_y < H) return OCC_EINVAL;
  struct {
    const void *w, *s;
    size_t stride, rows, cols;
  } m[3] = {{a.w_gate, a.s_gate, a.stride_gate, I, H}, {a.w_up, a.s_up, a.stride_up, I, H}, {a.w_down, a.s_down, a.stride_down, H, I}};
  Range in[9] = {{a.x, ((T - 1) * a.ld_x + H) * 2}, {a.router, E * H * 2}, {a.mask, T}};
  for (int i = 0; i < 3; ++i) {
    if (m[i].w == nullptr || !aligned(m[i].w, 16)) return OCC_EINVAL;
    if (mx) {
      if (m[i].s == nullptr || !aligned(m[i].s, 16) || m[i].stride != 0) return OCC_EINVAL;
      in[3 + 2 * i] = {m[i].w, E * OCC_MX4_CODE_BYTES(m[i].rows, m[i].cols)};
      in[4 + 2 * i] = {m[i].s, E * OCC_MX4_SCALE_BYTES(m[i].rows, m[i].cols)};
    } else {
      const size_t one = m[i].rows * m[i].cols, stride = m[i].stride == 0 ? one : m[i].stride;
      if (stride < one || stride % 8 != 0) return OCC_EINVAL;
      in[3 + 2 * i] = {m[i].w, ((E - 1) * stride + one) * 2};
      in[4 + 2 * i] = {nullptr, 0};
    }
  }
  const size_t need = moe_workspace(a.tokens, a.H, a.I, a.experts, a.top_k);
  if (a.workspace == nullptr || !aligned(a.workspace, 16) || a.workspace_bytes < need) return OCC_EINVAL;
  const Range out[] = {{a.y, ((T - 1) * a.ld_y + H) * 2}, {a.ids, T * k * 4}, {a.weights, T * k * 4}, {a.workspace, need}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

}  // namespace occ

extern "C" {

int occ_mx4_quantize(const void *x, int dtype, int rows, int cols, size_t ld, void *codes, void *scales,
                     void *codes_t, void *scales_t, void *stream) {
  const occ::Mx4QuantCall c{x, dtype, rows, cols, ld, codes, scales, codes_t, scales_t};
  const int st = occ::validate_mx4_quant(c);
  return st == OCC_OK ? occ::mx4_quant_launch(c, static_cast<hipStream_t>(stream)) : st;
}

int occ_mx4_dequantize(const void *codes, const void *scales, int rows, int cols, void *out, int dtype, size_t ld,
                       void *stream) {
  const occ::Mx4DequantCall c{codes, scales, rows, cols, out, dtype, ld};
  const int st = occ::validate_mx4_dequant(c);
  return st == OCC_OK ? occ::mx4_dequant_launch(c, static_cast<hipStream_t>(stream)) : st;
}

int occ_gemm_mx4(const void *A, const void *A_scales, const void *B, const void *B_scales, void *C, int dtype,
                 int M, int N, int K, size_t lds_bytes, void *stream) {
  const occ::Mx4GemmCall c{A, A_scales, B, B_scales, C, dtype, M, N, K, lds_bytes};
  const int st = occ::validate_mx4_gemm(c);
  return st == OCC_OK ? occ::mx4_gemm_launch(c, static_cast<hipStream_t>(stream)) : st;
}

int occ_gemm_mx4_plan_query(int M, int N, int K, int num_cus, occ_gemm_mx4_plan *plan) {
  if (plan == nullptr || num_cus < 0 || occ::validate_mx4_gemm_dims(M, N, K) != OCC_OK) return OCC_EINVAL;
  if (num_cus == 0) {
    const occ::DeviceInfo *di = nullptr;
    const int st = occ::current_device_info(&di);
    if (st != OCC_OK) return st;
    num_cus = di->num_cus;
  }
  occ::mx4_gemm_plan(M, N, K, num_cus, plan);
  return OCC_OK;
}

int occ_norm_gate(const occ_norm_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_norm(*args, false);
  return st == OCC_OK ? occ::norm_gate_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

int occ_norm_gate_bwd(const occ_norm_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_norm(*args, true);
  return st == OCC_OK ? occ::norm_gate_bwd_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

size_t occ_norm_gate_bwd_workspace_bytes(int rows, int D, int groups) {
  if (rows < 0 || D < 1 || D > OCC_NORM_MAX_D || groups < 1 || groups > (rows > 0 ? rows : 1)) return 0;
  return occ::norm_bwd_workspace(rows, D, groups);
}

int occ_moe(const occ_moe_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_moe(*args);
  return st == OCC_OK ? occ::moe_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

size_t occ_moe_workspace_bytes(int tokens, int H, int I, int experts, int top_k) {
  if (tokens == 0 || occ::validate_moe_sizes(tokens, H, I, experts, top_k) != OCC_OK) return 0;
  return occ::moe_workspace(tokens, H, I, experts, top_k);
}

}  // extern "C"
