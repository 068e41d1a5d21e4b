// C = A B^T of MX4 operands (occ_gemm_mx4): the tiles, and which call takes which.
//
// fp32 accumulation on v_mfma_scale_f32_16x16x128_f8f6f4: exact products of two
// E2M1 values and two powers of two, 128 a lane group and instruction.  The
// kernels live in gemm_mx4_pp.h (256x256 tiles), gemm_mx4_rp.h (smaller ones) and
// gemm_mx4_skinny.h (M <= 16).
#include "gemm_mx4_pp.h"
#include "gemm_mx4_rp.h"
#include "gemm_mx4_skinny.h"
#include "once.h"

#include <algorithm>
#include <cmath>

namespace occ {
namespace {

typedef void (*Mx4Fn)(Mx4Operands, int, int);

// A tile and its estimated time on a shape: rounds of up to per_cu workgroups a CU, each of them a
// fixed part and a step per 512 of K, in us, where the CUs are lightly loaded and where they are full.
struct Mx4Tile {
  int bm, bn, threads, lds;
  Mx4Fn bf16, f32;
  int per_cu;  // workgroups resident on a CU
  double fixed, step, full_fixed, full_step;
  // n tiles at once.  A full chip slows a tile of one workgroup a CU with what all CUs store and load
  // together and with its clock, which a part of it does little; one of two a CU from
  // where CUs have two.
  double round_us(double n, double num_cus, double k) const {
    const double x = per_cu == 2 ? std::max(0.0, n / num_cus - 1) : n / num_cus * (n / num_cus);
    return (1 - x) * (fixed + step * k) + x * (full_fixed + full_step * k);
  }
};

template <template <class> class T>
constexpr Mx4Tile tile_of(Mx4Fn bf16, Mx4Fn f32, int per_cu, double fixed, double step, double full_fixed, double full_step) {
  typedef T<uint16_t> X;
  return Mx4Tile{X::BM, X::BN, X::NT, X::LDS_BYTES, bf16, f32, per_cu, fixed, step, full_fixed, full_step};
}

template <class OUT>
using Rp128x128 = Mx4Rp<128, 128, 2, 2, 256, 2, 1, OUT>;
template <class OUT>
using Rp128x64 = Mx4Rp<128, 64, 4, 2, 512, 3, 2, OUT>;
template <class OUT>
using Rp64x64 = Mx4Rp<64, 64, 2, 2, 512, 4, 4, OUT>;
template <class OUT>
using Rp32x64 = Mx4Rp<32, 64, 2, 2, 512, 4, 4, OUT>;

// Fitted to shapes from 17 x 512 x 512 to 16384 x 8192 x 512.  They hold no bytes: where few rows read a large
// B once (64 x 28672 x 8192: 16 us by them, 31 measured, of which B's bytes are 21) every estimate is too low,
// and the choice rests on the tiles' order alone.  128x128 at two workgroups a CU passes 256x256 where K is short
// (16384 x 8192 x 512: 84 us, 92) or the larger tiles leave CUs idle (2500 x 2500 x 8192:
// 31, 46; 3001 x 2504 x 5003: 25, 33), and is passed by it on the large ones (8192^3: 269, 234).
const Mx4Tile kTiles[] = {
    tile_of<Mx4Pp>(gemm_mx4_pp_kernel<Mx4Pp<uint16_t>>, gemm_mx4_pp_kernel<Mx4Pp<float>>, 1, 4.0, 2.2, 9.0, 2.75),
    tile_of<Rp128x128>(gemm_mx4_rp_kernel<Rp128x128<uint16_t>>, gemm_mx4_rp_kernel<Rp128x128<float>>, 2, 1.5, 0.95, 3.1, 1.9),
    tile_of<Rp128x64>(gemm_mx4_rp_kernel<Rp128x64<uint16_t>>, gemm_mx4_rp_kernel<Rp128x64<float>>, 1, 1.8, 0.6, 1.8, 0.6),
    tile_of<Rp64x64>(gemm_mx4_rp_kernel<Rp64x64<uint16_t>>, gemm_mx4_rp_kernel<Rp64x64<float>>, 1, 1.6, 0.4, 1.6, 0.4),
    tile_of<Rp32x64>(gemm_mx4_rp_kernel<Rp32x64<uint16_t>>, gemm_mx4_rp_kernel<Rp32x64<float>>, 1, 1.3, 0.33, 1.3, 0.33),
};
constexpr int kMaxDevices = 64;
constexpr int kNumTiles = (int)(sizeof kTiles / sizeof kTiles[0]);

int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }

// The tile with the least estimated time.
int choose_tile(int M, int N, int K, int num_cus) {
  int best = -1;
  double t_best = 0;
  for (int i = 0; i < kNumTiles; ++i) {
    const Mx4Tile &t = kTiles[i];
    const double tiles = (double)ceil_div(M, t.bm) * ceil_div(N, t.bn);
    const double k = ceil_div(K, 512), slots = (double)t.per_cu * num_cus, rounds = std::floor(tiles / slots);
    const double us = rounds * t.round_us(slots, num_cus, k) + (tiles > rounds * slots ? t.round_us(tiles - rounds * slots, num_cus, k) : 0);
    if (best < 0 || us < t_best) {
      best = i;
      t_best = us;
    }
  }
  return best;
}

// A B that is read once and exceeds the eight 4 MB L2s goes past them.
constexpr long long kNtBytes = 32ll << 20;

typedef void (*SkinnyFn)(Mx4Operands, int);

template <class OUT>
SkinnyFn skinny_fn(int kw, int xs, bool nt) {
  if (xs == 2) return nt ? gemm_mx4_skinny_kernel<8, 2, OUT, true> : gemm_mx4_skinny_kernel<8, 2, OUT, false>;
  if (kw == 8) return nt ? gemm_mx4_skinny_kernel<8, 1, OUT, true> : gemm_mx4_skinny_kernel<8, 1, OUT, false>;
  return kw == 4 ? gemm_mx4_skinny_kernel<4, 1, OUT, false> : kw == 2 ? gemm_mx4_skinny_kernel<2, 1, OUT, false>
                                                                    : gemm_mx4_skinny_kernel<1, 1, OUT, false>;
}

// The pad's limit, once it is known to fit: an attribute that matters to pads only.
int allow_lds(const void *fn, size_t lds_bytes, int own, const DeviceInfo &di) {
  if ((size_t)own + lds_bytes > (size_t)di.max_lds_per_wg) return OCC_ELDS;
  if (lds_bytes == 0) return OCC_OK;
  return hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, di.max_lds_per_wg - own) == hipSuccess ? OCC_OK
                                                                                                                   : OCC_EHIP;
}

// Of a call with M <= 16.
struct SkinnyPlan {
  int kw, xs;  // waves along K, one a k-step, up to 8; k-steps of A that each keeps
  bool fits;   // A in registers
  bool nt;
  int units, grid;
};
SkinnyPlan skinny_plan(int N, int K, int num_cus) {
  SkinnyPlan p{};
  const int steps512 = ceil_div(K, 512);
  p.kw = 1;
  while (p.kw < 8 && p.kw < steps512) p.kw *= 2;
  p.xs = std::max(1, ceil_div(steps512, p.kw));
  p.fits = p.xs <= 2;
  p.nt = p.fits && p.kw == 8 && (long long)N * (long long)(OCC_MX4_KP(K) / 2) > kNtBytes;
  p.units = ceil_div(N, p.fits ? 16 : 32);
  p.grid = p.fits ? std::min(ceil_div(p.units, 8 / p.kw), 2 * num_cus) : p.units;
  return p;
}

int launch_skinny(const Mx4GemmCall &c, const Mx4Operands &o, const DeviceInfo &di, hipStream_t s) {
  const SkinnyPlan p = skinny_plan(c.N, c.K, di.num_cus);
  if (!p.fits) {
    typedef void (*LongFn)(Mx4Operands);
    const LongFn fn = c.dtype == OCC_BF16 ? gemm_mx4_skinny_long_kernel<uint16_t> : gemm_mx4_skinny_long_kernel<float>;
    const int st = allow_lds(reinterpret_cast<const void *>(fn), c.lds_bytes, 8 * 2 * 1024, di);
    if (st != OCC_OK) return st;
    hipLaunchKernelGGL(fn, dim3(p.grid), dim3(512), (int)c.lds_bytes, s, o);
    return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
  }
  const SkinnyFn fn = c.dtype == OCC_BF16 ? skinny_fn<uint16_t>(p.kw, p.xs, p.nt) : skinny_fn<float>(p.kw, p.xs, p.nt);
  const int st = allow_lds(reinterpret_cast<const void *>(fn), c.lds_bytes, 8 * 4096 + 16 * 1024, di);
  if (st != OCC_OK) return st;
  hipLaunchKernelGGL(fn, dim3(p.grid), dim3(512), (int)c.lds_bytes, s, o, p.units);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace

void mx4_gemm_plan(int M, int N, int K, int num_cus, occ_gemm_mx4_plan *plan) {
  *plan = occ_gemm_mx4_plan{};
  if (M == 0 || N == 0) return;
  if (M <= 16) {
    const SkinnyPlan p = skinny_plan(N, K, num_cus);
    *plan = occ_gemm_mx4_plan{16, p.fits ? 16 : 32, p.units, p.grid, p.nt};
    return;
  }
  const Mx4Tile &t = kTiles[choose_tile(M, N, K, num_cus)];
  const int tiles = ceil_div(M, t.bm) * ceil_div(N, t.bn);
  *plan = occ_gemm_mx4_plan{t.bm, t.bn, tiles, tiles, 0};
}

int mx4_gemm_launch(const Mx4GemmCall &c, hipStream_t s) {
  const DeviceInfo *di = nullptr;
  int st = current_device_info(&di);
  if (st != OCC_OK) return st;
  if (c.M == 0 || c.N == 0) return OCC_OK;
  const Mx4Operands o{static_cast<const uint8_t *>(c.A), static_cast<const uint8_t *>(c.As),
                      static_cast<const uint8_t *>(c.B), static_cast<const uint8_t *>(c.Bs),
                      c.C, c.M, c.N, (uint32_t)(OCC_MX4_KP(c.K) / 2), ceil_div(c.K, 256), ceil_div(c.K, 512)};
  if (c.M <= 16) return launch_skinny(c, o, *di, s);
  if (c.lds_bytes > (size_t)di->max_lds_per_wg) return OCC_ELDS;
  // the pad keeps the tile: it lowers residency and changes nothing else, and is never clamped
  const int id = choose_tile(c.M, c.N, c.K, di->num_cus);
  const Mx4Tile &t = kTiles[id];
  if ((size_t)t.lds + c.lds_bytes > (size_t)di->max_lds_per_wg) return OCC_ELDS;
  const Mx4Fn fn = c.dtype == OCC_BF16 ? t.bf16 : t.f32;
  // the dynamic-LDS limit is a per-device attribute of each kernel: set once
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return OCC_ENODEV;
  static Once attr_set[kMaxDevices][kNumTiles][2];
  if (!attr_set[dev][id][c.dtype == OCC_F32].run([&] {
        return hipFuncSetAttribute(reinterpret_cast<const void *>(fn), hipFuncAttributeMaxDynamicSharedMemorySize,
                                   di->max_lds_per_wg) == hipSuccess;
      }))
    return OCC_EHIP;
  const int tm = ceil_div(c.M, t.bm), tn = ceil_div(c.N, t.bn);
  hipLaunchKernelGGL(fn, dim3(tm * tn), dim3(t.threads), t.lds + (int)c.lds_bytes, s, o, tm, tn);
  return hipGetLastError() == hipSuccess ? OCC_OK : OCC_EHIP;
}

}  // namespace occ
