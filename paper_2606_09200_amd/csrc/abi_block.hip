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

namespace {

// Bytes that heads of D values at these pitches span.
size_t span3(int rows, size_t row, int heads, size_t head, int D, size_t elem) {
  return rows == 0 || heads == 0 ? 0 : ((size_t)(rows - 1) * row + (size_t)(heads - 1) * head + D) * elem;
}
// Heads that do not overlap, in rows that do not: one pitch goes past what the other covers.
bool apart(int rows, size_t row, int heads, size_t head, int D) {
  const size_t d = (size_t)D;
  if (heads > 1 && head < d) return false;
  if (rows > 1 && row < d) return false;
  if (heads <= 1 || rows <= 1) return true;
  return row >= (size_t)(heads - 1) * head + d || head >= (size_t)(rows - 1) * row + d;
}
// How many heads, rows and pages of D values there are, and how far apart (elements).
struct Pitches {
  int count[3];
  size_t pitch[3];
};
// Whether the values of x and y, in one buffer, are not each other's because of a period, one of their pitches: of what lies within
// it (heads in a row, say), x's begins behind y's end and ends within it, and all else is whole periods away.
bool interleaved(const void *x, const Pitches &gx, const void *y, const Pitches &gy, int D, size_t elem) {
  const uintptr_t px = reinterpret_cast<uintptr_t>(x), py = reinterpret_cast<uintptr_t>(y);
  auto within = [&](const Pitches &g, size_t period, size_t &width) {
    width = (size_t)D;
    for (int i = 0; i < 3; ++i) {
      if (g.count[i] <= 1) continue;
      if (g.pitch[i] < period) width += (size_t)(g.count[i] - 1) * g.pitch[i];
      else if (g.pitch[i] % period != 0) return false;
    }
    return true;
  };
  for (const Pitches *g : {&gx, &gy})
    for (int i = 0; i < 3; ++i) {
      if (g->count[i] <= 1 || g->pitch[i] == 0) continue;
      size_t wx, wy;
      if (!within(gx, g->pitch[i], wx) || !within(gy, g->pitch[i], wy)) continue;
      const size_t period = g->pitch[i] * elem, off = px >= py ? (px - py) % period : (period - (py - px) % period) % period;
      if (off >= wy * elem && off + wx * elem <= period) return true;
    }
  return false;
}
// The same of a cache's rows in pages; pages are outermost, then rows or heads.
bool cache_apart(int pages, size_t cache_page, int page, size_t row, int heads, size_t head, int D) {
  return apart(page, row, heads, head, D) && (pages <= 1 || cache_page >= span3(page, row, heads, head, D, 1));
}

}  // namespace

int validate_kv_tables(const occ_kv_tables_args &a) {
  if (a.requests < 0 || a.requests > OCC_KV_MAX_REQUESTS || a.rows < 0 || a.rows > (1 << 24)) return OCC_EINVAL;
  if (a.width < 0 || a.page < 1 || a.page > OCC_KV_MAX_PAGE || a.pages < 0 || a.ring_size < 1) return OCC_EINVAL;
  if ((long long)a.pages * a.page > INT32_MAX || a.ring_size > (1 << 30)) return OCC_EINVAL;
  if (a.requests > 1 && a.ld_table < (size_t)a.width) return OCC_EINVAL;
  const void *all[] = {a.cached, a.fresh, a.lens, a.table, a.free, a.ring, a.starts, a.free_after};
  for (const void *p : all)
    if (!aligned(p, 4)) return OCC_EINVAL;
  if (a.requests > 0 && (a.cached == nullptr || a.fresh == nullptr || a.lens == nullptr || (a.width > 0 && a.table == nullptr))) return OCC_EINVAL;
  if (a.free == nullptr || a.ring == nullptr || a.starts == nullptr || a.free_after == nullptr) return OCC_EINVAL;
  if (a.rows > 0 && (a.slots == nullptr || a.positions == nullptr)) return OCC_EINVAL;
  if (!aligned(a.slots, 4) || !aligned(a.positions, 4)) return OCC_EINVAL;
  const size_t n = (size_t)a.requests * 4, t = (size_t)a.rows * 4;
  const Range in[] = {{a.cached, n}, {a.fresh, n}, {a.free, 8}};
  const Range out[] = {{a.table, a.width == 0 || a.requests == 0 ? 0 : ((size_t)(a.requests - 1) * a.ld_table + a.width) * 4},
                       {a.ring, (size_t)a.ring_size * 4}, {a.lens, n}, {a.starts, n + 4}, {a.slots, t}, {a.positions, t},
                       {a.free_after, 8}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

int validate_rope(const occ_rope_args &a) {
  if (!float_type(a.dtype) || a.rows < 0 || a.rows > (1 << 24) || a.Hq < 0 || a.Hkv < 0) return OCC_EINVAL;
  if (a.Hq > 65536 || a.Hkv > 65536 || a.D < 2 || a.D > OCC_ROPE_MAX_D || a.D % 2 != 0) return OCC_EINVAL;
  if (a.pairs < 0 || a.pairs > a.D / 2 || !(a.scale - a.scale == 0.f)) return OCC_EINVAL;
  const bool cache = a.k_cache != nullptr;
  if (cache != (a.v_cache != nullptr)) return OCC_EINVAL;
  if (a.rows == 0) return OCC_OK;
  const size_t e = type_bytes(a.dtype);
  const bool q = a.q != nullptr && a.Hq > 0, k = a.k != nullptr && a.Hkv > 0;
  if (a.positions == nullptr || !aligned(a.positions, 4) || (a.pairs > 0 && a.turns == nullptr) || !aligned(a.turns, 8)) return OCC_EINVAL;
  if ((q && a.q_out == nullptr) || (k && a.k_out == nullptr && !cache) || (cache && (!k || a.v == nullptr || a.slots == nullptr)))
    return OCC_EINVAL;
  const void *all[] = {a.q, a.k, a.v, a.q_out, a.k_out, a.k_cache, a.v_cache};
  for (const void *p : all)
    if (!aligned(p, e)) return OCC_EINVAL;
  if (!aligned(a.slots, 4)) return OCC_EINVAL;
  if ((q && (!apart(a.rows, a.q_row, a.Hq, a.q_head, a.D) || !apart(a.rows, a.qo_row, a.Hq, a.qo_head, a.D))) ||
      (k && !apart(a.rows, a.k_row, a.Hkv, a.k_head, a.D)) ||
      (k && a.k_out != nullptr && !apart(a.rows, a.ko_row, a.Hkv, a.ko_head, a.D)))
    return OCC_EINVAL;
  if (cache && (a.page < 1 || a.page > OCC_KV_MAX_PAGE || a.pages < 1 || (long long)a.page * a.pages > INT32_MAX ||
                !apart(a.rows, a.v_row, a.Hkv, a.v_head, a.D) ||
                !cache_apart(a.pages, a.cache_page, a.page, a.cache_row, a.Hkv, a.cache_head, a.D)))
    return OCC_EINVAL;
  const Range rq{q ? a.q : nullptr, span3(a.rows, a.q_row, a.Hq, a.q_head, a.D, e)};
  const Range rk{k ? a.k : nullptr, span3(a.rows, a.k_row, a.Hkv, a.k_head, a.D, e)};
  const Range rv{cache ? a.v : nullptr, span3(a.rows, a.v_row, a.Hkv, a.v_head, a.D, e)};
  const Range qo{q ? a.q_out : nullptr, span3(a.rows, a.qo_row, a.Hq, a.qo_head, a.D, e)};
  const Range ko{k ? a.k_out : nullptr, span3(a.rows, a.ko_row, a.Hkv, a.ko_head, a.D, e)};
  const size_t cached = cache ? ((size_t)(a.pages - 1) * a.cache_page) * e + span3(a.page, a.cache_row, a.Hkv, a.cache_head, a.D, e) : 0;
  const Range kc{a.k_cache, cached}, vc{a.v_cache, cached};
  const Range pos{a.positions, (size_t)a.rows * 4}, turns{a.turns, (size_t)a.pairs * 8}, slots{cache ? a.slots : nullptr, (size_t)a.rows * 4};
  // q, k and v may lie among each other, as a joint projection leaves them, and so may keys and values of one cache
  const Pitches gq{{a.Hq, a.rows, 1}, {a.q_head, a.q_row, 0}}, gk{{a.Hkv, a.rows, 1}, {a.k_head, a.k_row, 0}};
  const Pitches gv{{a.Hkv, a.rows, 1}, {a.v_head, a.v_row, 0}}, gqo{{a.Hq, a.rows, 1}, {a.qo_head, a.qo_row, 0}};
  const Pitches gko{{a.Hkv, a.rows, 1}, {a.ko_head, a.ko_row, 0}};
  auto among = [&](const Range &x, const Pitches &gx, const Range &y, const Pitches &gy) {
    return !overlaps(x, y) || interleaved(x.p, gx, y.p, gy, a.D, e);
  };
  const bool same_q = a.q_out == a.q && a.qo_row == a.q_row && a.qo_head == a.q_head;
  const bool same_k = a.k_out == a.k && a.ko_row == a.k_row && a.ko_head == a.k_head;
  if (q && !same_q && !among(qo, gqo, rq, gq)) return OCC_EALIAS;
  if (q && k && !among(qo, gqo, rk, gk)) return OCC_EALIAS;
  if (q && cache && !among(qo, gqo, rv, gv)) return OCC_EALIAS;
  if (k && a.k_out != nullptr) {
    if (!same_k && !among(ko, gko, rk, gk)) return OCC_EALIAS;
    if (q && !among(ko, gko, rq, gq)) return OCC_EALIAS;
    if (q && !among(ko, gko, qo, gqo)) return OCC_EALIAS;
    if (cache && !among(ko, gko, rv, gv)) return OCC_EALIAS;
  }
  if (cache) {
    const Pitches g{{a.Hkv, a.page, a.pages}, {a.cache_head, a.cache_row, a.cache_page}};
    if (!among(kc, g, vc, g)) return OCC_EALIAS;
  }
  const Range in[] = {pos, turns, slots}, wide[] = {rq, rk, rv};
  const Range out[] = {kc};
  const Range out_v[] = {vc};
  for (const Range &o : {qo, ko, kc, vc})
    for (const Range &i : in)
      if (overlaps(o, i)) return OCC_EALIAS;
  if (!disjoint(out, wide) || !disjoint(out_v, wide)) return OCC_EALIAS;
  for (const Range &c : {kc, vc})
    if (overlaps(c, qo) || overlaps(c, ko)) return OCC_EALIAS;
  return OCC_OK;
}

bool attn_heads(int Hq, int Hkv, int D) {
  return Hkv >= 1 && Hq >= Hkv && Hq <= 65536 && Hq % Hkv == 0 && D >= 8 && D <= 256 && D % 8 == 0;
}

int validate_attn(const occ_attn_args &a) {
  if (!attn_heads(a.Hq, a.Hkv, a.D)) return OCC_EINVAL;
  if (a.requests < 0 || a.requests > OCC_KV_MAX_REQUESTS || a.rows < 0 || (long long)a.rows * a.Hq > INT32_MAX) return OCC_EINVAL;
  if (a.page < 1 || a.page > OCC_KV_MAX_PAGE || a.width < 0 || a.max_fresh < 0 || a.window < 0) return OCC_EINVAL;
  if (!(a.scale > 0.f && a.scale <= 0x1p127f)) return OCC_EINVAL;  // the kernels' is log2 e times that
  if (a.requests == 0 || a.rows == 0) return OCC_OK;
  if (a.pages < 1 || (long long)a.pages * a.page > INT32_MAX) return OCC_EINVAL;
  const void *wide[] = {a.q, a.k_cache, a.v_cache, a.out, a.workspace};
  for (const void *p : wide)
    if (p == nullptr || !aligned(p, 16)) return OCC_EINVAL;
  if (a.starts == nullptr || a.lens == nullptr || (a.width > 0 && a.table == nullptr)) return OCC_EINVAL;
  if (!aligned(a.starts, 4) || !aligned(a.lens, 4) || !aligned(a.table, 4) || !aligned(a.lse, 4)) return OCC_EINVAL;
  if ((a.q_row | a.q_head | a.out_row | a.out_head | a.cache_page | a.cache_row | a.cache_head) % 8 != 0) return OCC_EINVAL;
  if (a.requests > 1 && a.ld_table < (size_t)a.width) return OCC_EINVAL;
  if (!apart(a.rows, a.q_row, a.Hq, a.q_head, a.D) || !apart(a.rows, a.out_row, a.Hq, a.out_head, a.D)) return OCC_EINVAL;
  if (!cache_apart(a.pages, a.cache_page, a.page, a.cache_row, a.Hkv, a.cache_head, a.D)) return OCC_EINVAL;
  // pitches are 32-bit numbers in the kernels, units of work 64-bit ones with some bits to spare
  if ((a.pages > 1 && a.cache_page > OCC_ATTN_MAX_PITCH) || (a.page > 1 && a.cache_row > OCC_ATTN_MAX_PITCH)) return OCC_EINVAL;
  if (((double)a.rows + a.requests) * a.width * a.page * a.Hq >= 0x1p50) return OCC_EINVAL;
  const size_t need = attn_workspace(a.D);
  if (a.workspace_bytes < need) return OCC_EINVAL;
  const size_t cached = (size_t)(a.pages - 1) * a.cache_page * 2 + span3(a.page, a.cache_row, a.Hkv, a.cache_head, a.D, 2);
  const Range in[] = {{a.q, span3(a.rows, a.q_row, a.Hq, a.q_head, a.D, 2)}, {a.k_cache, cached}, {a.v_cache, cached},
                      {a.table, a.width == 0 ? 0 : ((size_t)(a.requests - 1) * a.ld_table + a.width) * 4},
                      {a.starts, (size_t)(a.requests + 1) * 4}, {a.lens, (size_t)a.requests * 4}};
  const Range out[] = {{a.out, span3(a.rows, a.out_row, a.Hq, a.out_head, a.D, 2)}, {a.lse, (size_t)a.rows * a.Hq * 4}, {a.workspace, need}};
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

int occ_kv_tables(const occ_kv_tables_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_kv_tables(*args);
  return st == OCC_OK ? occ::kv_tables_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

int occ_rope(const occ_rope_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_rope(*args);
  return st == OCC_OK ? occ::rope_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

int occ_attn_paged(const occ_attn_args *args, void *stream) {
  if (args == nullptr) return OCC_EINVAL;
  const int st = occ::validate_attn(*args);
  return st == OCC_OK ? occ::attn_launch(*args, static_cast<hipStream_t>(stream)) : st;
}

size_t occ_attn_paged_workspace_bytes(int Hq, int Hkv, int D) {
  return occ::attn_heads(Hq, Hkv, D) ? occ::attn_workspace(D) : 0;
}

}  // extern "C"
