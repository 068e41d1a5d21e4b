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

int current_device() {
  const DeviceInfo *di = nullptr;
  return current_device_info(&di);
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

int validate_mx4_gemm(const Mx4GemmCall &c) {
  if (!float_type(c.dtype) || !mx4_dims(c.M, c.N) || !mx4_dims(c.M, c.K)) return OCC_EINVAL;
  if (c.M == 0 || c.N == 0) return OCC_OK;
  // the grid of the smallest tile (32 x 64) in work-items, as above
  if (((c.M + 31ull) / 32) * ((c.N + 63ull) / 64) >= (1ull << 23)) return OCC_EINVAL;
  if (c.C == nullptr || !aligned(c.C, type_bytes(c.dtype))) return OCC_EINVAL;
  if (c.K > 0 && (!mx4_pointers(c.A, c.As) || !mx4_pointers(c.B, c.Bs))) return OCC_EINVAL;
  const Range in[] = {{c.A, OCC_MX4_CODE_BYTES(c.M, c.K)}, {c.As, OCC_MX4_SCALE_BYTES(c.M, c.K)},
                      {c.B, OCC_MX4_CODE_BYTES(c.N, c.K)}, {c.Bs, OCC_MX4_SCALE_BYTES(c.N, c.K)}};
  const Range out[] = {{c.C, span(c.M, c.N, c.N, c.dtype)}};
  return disjoint(out, in) ? OCC_OK : OCC_EALIAS;
}

}  // namespace occ

extern "C" {

int occ_mx4_quantize(const void *x, int dtype, int rows, int cols, size_t ld, void *codes, void *scales,
                     void *codes_t, void *scales_t, void *stream) {
  const occ::Mx4QuantCall c{x, dtype, rows, cols, ld, codes, scales, codes_t, scales_t};
  int st = occ::validate_mx4_quant(c);
  if (st == OCC_OK) st = occ::current_device();
  return st == OCC_OK ? occ::mx4_quant_launch(c, static_cast<hipStream_t>(stream)) : st;
}

int occ_mx4_dequantize(const void *codes, const void *scales, int rows, int cols, void *out, int dtype, size_t ld,
                       void *stream) {
  const occ::Mx4DequantCall c{codes, scales, rows, cols, out, dtype, ld};
  int st = occ::validate_mx4_dequant(c);
  if (st == OCC_OK) st = occ::current_device();
  return st == OCC_OK ? occ::mx4_dequant_launch(c, static_cast<hipStream_t>(stream)) : st;
}

int occ_gemm_mx4(const void *A, const void *A_scales, const void *B, const void *B_scales, void *C, int dtype,
                 int M, int N, int K, size_t lds_bytes, void *stream) {
  const occ::Mx4GemmCall c{A, A_scales, B, B_scales, C, dtype, M, N, K, lds_bytes};
  const int st = occ::validate_mx4_gemm(c);
  return st == OCC_OK ? occ::mx4_gemm_launch(c, static_cast<hipStream_t>(stream)) : st;
}

}  // extern "C"
