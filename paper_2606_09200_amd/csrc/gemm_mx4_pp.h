// Large-tile MX4 GEMM (included by gemm_mx4.hip only).
#pragma once

#include "gemm_mx4_common.h"

namespace occ {
namespace {

// ---------------------------------------------------------------------------
// 256 x 256 output tile, k-steps of 256 (128 bytes of codes a row), 8 waves, two LDS
// stages and one workgroup per CU: the schedule of gemm_pp.h, whose operand bytes,
// LDS layout and MFMA count per k-step are the same with 4 bits a value and 128
// deep MFMAs (16x16x128, as many cycles as 16x16x32 of bf16).  What differs:
//
//  * Scales.  A scale tile (16 rows x 512 columns, 256 bytes) is the operand of four
//    MFMAs: lane l's word holds its row's scale in each of the four 128-wide
//    steps, picked by the instruction's byte select.  Every second k-step, one
//    DMA per wave fetches the next super-step's 32 tiles (8 KiB, 4 tiles a wave,
//    1 KiB of contiguous 256-byte pieces); a phase reads the 4 words it needs of A
//    and, first in a k-step, of B.
//  * Waits.  The scale DMA is issued first in the second phase of even k-steps, so up
//    to 9 DMAs instead of 8 are younger than what the next two waits need.
//
// K is padded by the format: rows of codes have whole 512-column pieces of zeros.
//
// 8192^3: 234 to 260 us, 4.2 to 4.7 PFLOP/s; K = 32768: 5.1.  Two bounds multiply.  Power: near the board's cap the
// clock is 1.84 GHz (operands of zeros run at 2.39, 1.33 times as fast).  And at either clock the matrix
// pipes are 58 % busy: the reads and barriers between the phases (with a quarter of the MFMAs the loop still
// takes two thirds of its time; LDS itself is 30 % busy) and a tile's first loads and last stores, 10 us of
// 60.  Memory is no bound: with every k-step in the L2 it gains 3 %.
template <class OUT>
struct Mx4Pp {
  typedef OUT Out;
  static constexpr int BM = 256, BN = 256, BK = 256, NT = 512;
  static constexpr int PART_BYTES = 128 * BK / 2;   // 128 rows of a k-step
  static constexpr int STAGE_BYTES = 4 * PART_BYTES;
  static constexpr int SCALE_BYTES = 32 * 256;      // 16 tiles of A, then 16 of B
  static constexpr int LDS_BYTES = 2 * STAGE_BYTES + 2 * SCALE_BYTES;
};

template <class T>
__global__ __launch_bounds__(T::NT) void gemm_mx4_pp_kernel(Mx4Operands o, int tiles_m, int tiles_n) {
  extern __shared__ __align__(16) unsigned char smem[];  // two stages, two scale areas, then the unused pad
  const int M = o.M, N = o.N;
  const uint32_t P = o.pitch;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = wave >> 2;  // which half of the waves; rows 64*half .. of A0 and of A1
  const int wn = wave & 3;     // columns 32*wn .. of B0 and of B1
  const int l16 = lane & 15, g = lane >> 4;
  const int ntiles = tiles_m * tiles_n;
  const int nk = o.steps256;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)smem;
  const uint32_t wave_lds = (uint32_t)wave * 1024u;

  const int r_in = threadIdx.x >> 3;
  const uint32_t lane_off = (uint32_t)r_in * P + 16u * (uint32_t)swz<8>(r_in, threadIdx.x & 7);
  const uint32_t pass_step = 64u * P;
  const uint32_t sc_off = (uint32_t)((wave & 3) * 4 + g) * P + (uint32_t)l16 * 16u;  // this lane's 16 bytes of a tile

  // LDS offset of a 16-row operand block's read, first 128 columns; the second's is ^ 64
  const int rd0 = l16 * 128 + swz<8>(l16, g) * 16;
  const int a_first = half * 64 * 128, b_first = 2 * T::PART_BYTES + wn * 32 * 128;  // uniform

  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, ntiles), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM;
  const int n0 = tn * T::BN;
  const uint32_t a_bytes = (uint32_t)min(T::BM, M - m0) * P;
  const uint32_t b_bytes = (uint32_t)min(T::BN, N - n0) * P;
  const uint8_t *Am = o.A + (size_t)m0 * P;
  const uint8_t *Bn = o.B + (size_t)n0 * P;
  // this wave's scale tiles: waves 0-3 fetch A's, 4-7 B's
  const uint8_t *Sw = half ? o.Bs + (size_t)(n0 >> 4) * P : o.As + (size_t)(m0 >> 4) * P;
  const uint32_t s_bytes = (uint32_t)min(16, ((half ? N - n0 : M - m0) + 15) >> 4) * P;
  auto issue = [&](int kt, int p) {
    const uint32_t k0 = (uint32_t)kt * 128u;
    const uint32_t slot = lds0 + (uint32_t)(kt & 1) * T::STAGE_BYTES + (uint32_t)p * T::PART_BYTES + wave_lds;
    const i32x4 rs = make_rsrc((p >= 2 ? Bn : Am) + k0, kt < nk ? (p >= 2 ? b_bytes : a_bytes) - k0 : 0u);
    const uint32_t v = lane_off + (uint32_t)(p & 1) * 2u * pass_step;
    lds_dma16(rs, slot, v);
    lds_dma16(rs, slot + 8192u, v + pass_step);
  };
  auto issue_scales = [&](int sp) {
    const uint32_t k0 = (uint32_t)sp * 256u;
    const i32x4 rs = make_rsrc(Sw + k0, 2 * sp < nk ? s_bytes - k0 : 0u);
    lds_dma16(rs, lds0 + 2u * T::STAGE_BYTES + (uint32_t)(sp & 1) * T::SCALE_BYTES + wave_lds, sc_off);
  };

  f32x4 acc[2][4][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[h][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  u32x4 af[2][4], bf[2][4];
  int as[4], bs[4];
  auto read_a = [&](const unsigned char *cur, const unsigned char *sc, int h) {
    int rd = rd0;
    asm volatile("" : "+v"(rd));  // the sums below are made here, not kept in registers over the loop
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        af[ks][i] = *reinterpret_cast<const u32x4 *>(cur + a_first + (rd ^ (ks * 64)) + h * T::PART_BYTES + i * 2048);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      as[i] = *reinterpret_cast<const int *>(sc + (h * 8 + half * 4 + i) * 256 + lane * 4);
  };
  auto read_b = [&](const unsigned char *cur, const unsigned char *sc) {
    int rd = rd0;
    asm volatile("" : "+v"(rd));
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
          bf[ks][2 * h + j] = *reinterpret_cast<const u32x4 *>(cur + b_first + (rd ^ (ks * 64)) + h * T::PART_BYTES + j * 2048);
        bs[2 * h + j] = *reinterpret_cast<const int *>(sc + (16 + h * 8 + wn * 2 + j) * 256 + lane * 4);
      }
  };
  auto multiply = [&](int h, auto odd) {  // odd: second k-step of its 512 columns, scale bytes 2 and 3
    constexpr int q = decltype(odd)::value ? 2 : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[h][i][j] = mfma_mx4<q>(bf[0][j], af[0][i], acc[h][i][j], bs[j], as[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[h][i][j] = mfma_mx4<q + 1>(bf[1][j], af[1][i], acc[h][i][j], bs[j], as[i]);
  };
  auto barrier = [&]() {  // nothing moves across it
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](int kt, auto odd) {
    constexpr bool ODD = decltype(odd)::value;
    const unsigned char *cur = smem + (ODD ? T::STAGE_BYTES : 0);
    const unsigned char *sc = smem + 2 * T::STAGE_BYTES + ((kt >> 1) & 1) * T::SCALE_BYTES;
    read_a(cur, sc, 0);
    read_b(cur, sc);
    issue(kt + 1, 1);
    wait_vmcnt<ODD ? 9 : 8>();
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    barrier();
    multiply(0, odd);
    barrier();
    read_a(cur, sc, 1);
    if constexpr (!ODD) issue_scales((kt >> 1) + 1);
    issue(kt + 2, 0); issue(kt + 2, 2); issue(kt + 2, 3);
    wait_vmcnt<ODD ? 8 : 9>();
    __builtin_amdgcn_s_waitcnt(0xC07F);
    barrier();
    multiply(1, odd);
    barrier();
  };

  issue_scales(0);
  issue(0, 0); issue(0, 2); issue(0, 3);
  issue(0, 1);
  issue(1, 0); issue(1, 2); issue(1, 3);
  wait_vmcnt<8>();
  barrier();
  if (half == 1) barrier();
  int kt = 0;
  for (; kt + 1 < nk; kt += 2) {
    step(kt, std::false_type{});
    step(kt + 1, std::true_type{});
  }
  if (kt < nk) step(kt, std::false_type{});
  if (half == 0) barrier();
  wait_vmcnt<0>();  // the DMA issued past the last k-step, before the stages get other use
  barrier();

  typedef TileOut<T::BN, typename T::Out> Out;
  static_assert(128 * Out::PITCH <= T::LDS_BYTES, "half a tile of C");
  int el = lane;
  asm volatile("" : "+v"(el));  // keeps the addresses below out of the k-loop's registers
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        Out::put(smem, half * 64 + i * 16, (j >> 1) * 128 + wn * 32 + (j & 1) * 16, el, acc[h][i][j]);
    __syncthreads();
    Out::template store<128, T::NT>(smem, static_cast<typename T::Out *>(o.C), M, N, m0 + h * 128, n0);
    if (h == 0) __syncthreads();
  }
}

}  // namespace
}  // namespace occ
