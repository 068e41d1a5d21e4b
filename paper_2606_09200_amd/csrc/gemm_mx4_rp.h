// Register-pipelined MX4 GEMM tiles smaller than 256x256 (included by gemm_mx4.hip only).
#pragma once

#include "gemm_mx4_common.h"

namespace occ {
namespace {

// One 4-byte-per-lane DMA into LDS at M0 + 4*lane (as lds_dma16).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma4(i32x4 rsrc, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// ---------------------------------------------------------------------------
// k-steps of 512 (256 bytes of codes a row, one scale tile per 16 rows), STAGES of
// them in LDS; the schedule of gemm_rp.h: a wave holds two sets of operand
// fragments, the MFMAs of one group of 128-wide substeps run while the next
// group's fragments are read and a later k-step's DMA is issued, and a k-step has
// one barrier, before its last group.  Scale tiles are fetched 256 bytes per
// DMA and read as one word per 16 rows and k-step, with the k-step's first group.
// BK = 256 halves the k-steps: rows of 128 bytes, each scale tile fetched with both
// steps that use it (four tiles per DMA), so that two workgroups share a CU.
// One's first loads and last stores then pass beside the other's products (128x128 with eight
// waves, k-steps of 512 and a CU to itself: 3001 x 2504 x 5003 30 us, now 25; 2500 x 2500 x 8192 41,
// now 31).  At 8192^3 it takes 15 % longer than the 256x256 tile, which reads a quarter less from LDS
// for the same MFMAs.
template <int BM_, int BN_, int WM_, int WN_, int BK_, int STAGES_, int GS_, class OUT>
struct Mx4Rp {
  typedef OUT Out;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, GS = GS_, BK = BK_;
  static constexpr int ROW = BK / 2, KS = BK / 128;  // bytes of a row, 128-wide substeps of a k-step
  static constexpr bool HALF = BK == 256;            // a k-step is half a scale tile
  static constexpr int WAVES = WM * WN, NT = 64 * WAVES;
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int CHUNKS = ROW / 16, RPP = NT / CHUNKS;  // 16-byte chunks of a row, rows per DMA pass
  static constexpr int A_LOADS = BM / RPP, B_LOADS = BN / RPP;
  static constexpr int TILES = (BM + BN) / 16;      // scale tiles
  static constexpr int S_LOADS = HALF ? TILES / 4 / WAVES : (TILES + WAVES - 1) / WAVES;
  static constexpr int LOADS = A_LOADS + B_LOADS + S_LOADS;
  static constexpr int A_BYTES = BM * ROW, CODE_BYTES = A_BYTES + BN * ROW;
  static constexpr int STAGE_BYTES = CODE_BYTES + S_LOADS * WAVES * (HALF ? 1024 : 256);
  static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
  static constexpr int NG = KS / GS;                // fragment groups per k-step
  static_assert(KS % GS == 0 && (NG == 1 || NG % 2 == 0), "groups alternate between two register sets");
  static_assert(BM % RPP == 0 && BN % RPP == 0 && RPP % 16 == 0, "uneven load passes, or a swizzle that changes between them");
  static_assert(BK == 512 || (HALF && BM % (64 * S_LOADS) == 0 && TILES == 4 * WAVES * S_LOADS && NG % 2 == 0),
                "a wave's scale DMA is of one operand's tiles");
  static_assert((STAGES - 1) * LOADS <= 63, "vmcnt holds at most 63");
};

// Chunk c of row r of a staged operand lies at (and the chunk there is) this one of the row.
template <class T>
__device__ __forceinline__ int mx4_rp_chunk(int r, int c) {
  if constexpr (T::HALF) return swz<8>(r, c);
  else return c ^ (r & 15);
}

template <class T>
__global__ __launch_bounds__(T::NT, 2) void gemm_mx4_rp_kernel(Mx4Operands o, int tiles_m, int tiles_n) {
  extern __shared__ __align__(16) unsigned char smem[];  // tile stages, then the unused pad
  constexpr int S = T::STAGES;
  const int M = o.M, N = o.N;
  const uint32_t P = o.pitch;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int l16 = lane & 15, g = lane >> 4;
  const int ntiles = tiles_m * tiles_n;
  const int nk = T::HALF ? o.steps256 : o.steps512;
  const uint32_t lds0 = (uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)smem;
  const uint32_t wave_lds = (uint32_t)wave * 1024u;

  // DMA slots: chunks spread by the row (the same in every pass)
  const int r_in = threadIdx.x / T::CHUNKS;
  const uint32_t lane_off = (uint32_t)r_in * P + 16u * (uint32_t)mx4_rp_chunk<T>(r_in, threadIdx.x % T::CHUNKS);
  const uint32_t pass_step = (uint32_t)T::RPP * P;

  int a_rd[T::KS], b_rd[T::KS];
#pragma unroll
  for (int ks = 0; ks < T::KS; ++ks) {
    a_rd[ks] = (wm * T::FM * 16 + l16) * T::ROW + mx4_rp_chunk<T>(l16, ks * 4 + g) * 16;
    b_rd[ks] = T::A_BYTES + (wn * T::FN * 16 + l16) * T::ROW + mx4_rp_chunk<T>(l16, ks * 4 + g) * 16;
  }

  int tm, tn;
  tile_coords<8>(xcd_remap(blockIdx.x, ntiles), tiles_m, tiles_n, tm, tn);
  const int m0 = tm * T::BM;
  const int n0 = tn * T::BN;
  const uint32_t a_bytes = (uint32_t)min(T::BM, M - m0) * P, b_bytes = (uint32_t)min(T::BN, N - n0) * P;
  const uint8_t *Am = o.A + (size_t)m0 * P, *Bn = o.B + (size_t)n0 * P;
  const uint8_t *Sa = o.As + (size_t)(m0 >> 4) * P, *Sb = o.Bs + (size_t)(n0 >> 4) * P;
  const int at = min(T::BM / 16, (M - m0 + 15) >> 4), bt = min(T::BN / 16, (N - n0 + 15) >> 4);  // tiles that exist
  // DMA pass p of k-step kt (A's, B's, then scales) into stage `slot`
  auto issue_pass = [&](int kt, uint32_t slot, int p) {
    const uint32_t k0 = (uint32_t)kt * T::ROW;
    const bool in = kt < nk;
    if (p < T::A_LOADS) {
      const i32x4 rs = make_rsrc(Am + k0, in ? a_bytes - k0 : 0u);
      lds_dma16(rs, slot + wave_lds + (uint32_t)(p * T::NT * 16), lane_off + (uint32_t)p * pass_step);
    } else if (p < T::A_LOADS + T::B_LOADS) {
      const int q = p - T::A_LOADS;
      const i32x4 rs = make_rsrc(Bn + k0, in ? b_bytes - k0 : 0u);
      lds_dma16(rs, slot + wave_lds + (uint32_t)(T::A_BYTES + q * T::NT * 16), lane_off + (uint32_t)q * pass_step);
    } else if constexpr (T::HALF) {
      const int x = ((p - T::A_LOADS - T::B_LOADS) * T::WAVES + wave) * 4;  // first of four scale tiles, A's then B's
      const bool b = x >= T::BM / 16;
      const uint32_t y = (uint32_t)(b ? x - T::BM / 16 : x), s0 = (uint32_t)(kt >> 1) * 256u;
      const i32x4 rs = make_rsrc((b ? Sb : Sa) + s0, in ? (uint32_t)(b ? bt : at) * P - s0 : 0u);
      lds_dma16(rs, slot + (uint32_t)(T::CODE_BYTES + x * 256), (y + g) * P + (uint32_t)l16 * 16u);
    } else {
      const int x = (p - T::A_LOADS - T::B_LOADS) * T::WAVES + wave;  // scale tile, A's then B's
      const bool b = x >= T::BM / 16;
      const int y = b ? x - T::BM / 16 : x;
      const bool exists = in && y < (b ? bt : at);
      const i32x4 rs = make_rsrc((b ? Sb : Sa) + (exists ? (size_t)y * P + k0 : 0), exists ? 256u : 0u);
      lds_dma4(rs, slot + (uint32_t)(T::CODE_BYTES + x * 256), (uint32_t)lane * 4u);
    }
  };

  f32x4 acc[T::FM][T::FN];
#pragma unroll
  for (int i = 0; i < T::FM; ++i)
#pragma unroll
    for (int j = 0; j < T::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  u32x4 af[2][T::GS][T::FM], bf[2][T::GS][T::FN];
  int as[T::FM], bs[T::FN], as_next[T::FM], bs_next[T::FN];
  constexpr int NR = T::GS * (T::FM + T::FN);   // fragments of a group
  constexpr int NM = T::GS * T::FM * T::FN;     // MFMAs of a group
  auto read_frag = [&](const unsigned char *cur, int gi, int set, int x) {
    const int s = x / (T::FM + T::FN), y = x % (T::FM + T::FN), ks = gi * T::GS + s;
    if (y < T::FM) af[set][s][y] = *reinterpret_cast<const u32x4 *>(cur + a_rd[ks] + y * 16 * T::ROW);
    else bf[set][s][y - T::FM] = *reinterpret_cast<const u32x4 *>(cur + b_rd[ks] + (y - T::FM) * 16 * T::ROW);
  };
  auto read_scales = [&](const unsigned char *cur) {
    const unsigned char *sc = cur + T::CODE_BYTES + lane * 4;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) as_next[i] = *reinterpret_cast<const int *>(sc + (wm * T::FM + i) * 256);
#pragma unroll
    for (int j = 0; j < T::FN; ++j)
      bs_next[j] = *reinterpret_cast<const int *>(sc + (T::BM / 16 + wn * T::FN + j) * 256);
  };
  auto mfma = [&](int byte0, int gi, int set, int x) {
    const int s = x / (T::FM * T::FN), i = x / T::FN % T::FM, j = x % T::FN;
    switch (byte0 + gi * T::GS + s) {  // a constant once unrolled
      case 0: acc[i][j] = mfma_mx4<0>(bf[set][s][j], af[set][s][i], acc[i][j], bs[j], as[i]); break;
      case 1: acc[i][j] = mfma_mx4<1>(bf[set][s][j], af[set][s][i], acc[i][j], bs[j], as[i]); break;
      case 2: acc[i][j] = mfma_mx4<2>(bf[set][s][j], af[set][s][i], acc[i][j], bs[j], as[i]); break;
      default: acc[i][j] = mfma_mx4<3>(bf[set][s][j], af[set][s][i], acc[i][j], bs[j], as[i]); break;
    }
  };
  auto slot_of = [&](int s) { return lds0 + (uint32_t)s * T::STAGE_BYTES; };
  auto publish = [&]() {  // this wave's reads are done; then every wave's, and its DMA has landed
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };

#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int p = 0; p < T::LOADS; ++p) issue_pass(s, slot_of(s), p);
  wait_vmcnt<(S - 1) * T::LOADS>();
  publish();
  read_scales(smem);
#pragma unroll
  for (int x = 0; x < NR; ++x) read_frag(smem, 0, 0, x);
  int stage = 0;  // stage of the k-step being multiplied
  auto step = [&](int kt, int set0, int byte0) {
    const int next = stage + 1 == S ? 0 : stage + 1;
    const unsigned char *cur = smem + stage * T::STAGE_BYTES, *nxt = smem + next * T::STAGE_BYTES;
    const uint32_t slot = slot_of(stage);
#pragma unroll
    for (int i = 0; i < T::FM; ++i) as[i] = as_next[i];
#pragma unroll
    for (int j = 0; j < T::FN; ++j) bs[j] = bs_next[j];
#pragma unroll
    for (int gi = 0; gi < T::NG; ++gi) {
      const int set = (set0 + gi) & 1;
      const bool last = gi + 1 == T::NG;
      if (last) {
        wait_vmcnt<(S - 2) * T::LOADS>();
        publish();
        read_scales(nxt);
      }
#pragma unroll
      for (int x = 0; x < NM; ++x) {
        mfma(byte0, gi, set, x);
        // the reads behind the first half of the MFMAs, the DMA behind all of them
#pragma unroll
        for (int y = 0; y < NR; ++y)
          if (y * (NM / 2) / NR == x) read_frag(last ? nxt : cur, last ? 0 : gi + 1, set ^ 1, y);
#pragma unroll
        for (int p = 0; p < T::LOADS; ++p)
          if (last && p * NM / T::LOADS == x) issue_pass(kt + S, slot, p);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    stage = next;
  };
  if constexpr (T::NG == 1 || T::HALF) {  // the register sets or the scales' bytes alternate
    int kt = 0;
    for (; kt + 1 < nk; kt += 2) {
      step(kt, 0, 0);
      step(kt + 1, T::NG == 1, T::HALF ? 2 : 0);
    }
    if (kt < nk) step(kt, 0, 0);
  } else {
    for (int kt = 0; kt < nk; ++kt) step(kt, 0, 0);
  }
  wait_vmcnt<0>();  // the DMA issued past the last k-step, before the stages get other use
  publish();

  typedef TileOut<T::BN, typename T::Out> Out;
  static_assert(T::BM * Out::PITCH <= T::LDS_BYTES, "a tile of C");
  int el = lane;
  asm volatile("" : "+v"(el));  // keeps the addresses below out of the k-loop's registers
#pragma unroll
  for (int i = 0; i < T::FM; ++i)
#pragma unroll
    for (int j = 0; j < T::FN; ++j) Out::put(smem, (wm * T::FM + i) * 16, (wn * T::FN + j) * 16, el, acc[i][j]);
  __syncthreads();
  Out::template store<T::BM, T::NT>(smem, static_cast<typename T::Out *>(o.C), M, N, m0, n0);
}

}  // namespace
}  // namespace occ
