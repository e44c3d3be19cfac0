// Core of the large bf16 products, for the files that bring epilogues of their own to it.
#pragma once

#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "hero_device.h"

namespace hero {
namespace {

constexpr int BK = 64;     // k elements per tile
constexpr int ROWB = 128;  // bytes of one row of a bf16 k-tile

template <typename T>
struct ARows {
  const T* base;
  const int* idx;  // null: identity
  int ld;
  // products of two terms (an epilogue with kTwoTerm): the operand from k-tile `turn` on, where B
  // starts over
  const T* base2 = nullptr;
  int turn = 0;
  // products of three-term operands (an epilogue with kSixTerm): elements from one term to the next;
  // `turn` k-tiles a term
  size_t term = 0;
  __device__ __forceinline__ const T* row(int m) const {
    return base + static_cast<size_t>(idx ? idx[m] : m) * ld;
  }
};

// B rows: [0, split) from b0, [split, ...) from b1 (router: W_hd then psi_1);
// for the gate/up product b0 = W_g, b1 = W_u and rows are addressed by column.
template <typename T>
struct BRows {
  const T* b0;
  const T* b1;
  int split;
  int ld;
  // the large products: rows past the last one repeat it, and rows may be gathered
  int last = INT_MAX;
  const int* idx = nullptr;
  size_t term = 0;   // as in ARows
  __device__ __forceinline__ const T* row(int n) const {
    return n < split ? b0 + static_cast<size_t>(n) * ld : b1 + static_cast<size_t>(n - split) * ld;
  }
  __device__ __forceinline__ const T* gate_row(int c) const { return b0 + static_cast<size_t>(c) * ld; }
  __device__ __forceinline__ const T* up_row(int c) const { return b1 + static_cast<size_t>(c) * ld; }
};

struct EpiStoreF32 {  // P[m][n] = acc; the MFMA path's K-slice z writes out + z * split_stride
  float* out;
  int ld;
  size_t split_stride;
  struct Pre {};
  __device__ __forceinline__ Pre prep(int, int) const { return {}; }
  __device__ __forceinline__ void store(int m, int n, float v) const {
    out[static_cast<size_t>(m) * ld + n] = v;
  }
  __device__ __forceinline__ void emit8(const Pre&, int m, int n, const float* v) const {
    float* o = out + blockIdx.y * split_stride + static_cast<size_t>(m) * ld + n;
    *reinterpret_cast<f32x4*>(o) = *reinterpret_cast<const f32x4*>(v);
    *reinterpret_cast<f32x4*>(o + 4) = *reinterpret_cast<const f32x4*>(v + 4);
  }
};

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ void load_lds16(const void* g, unsigned char* l) {
  __builtin_amdgcn_global_load_lds(g, (lds_void*)(l), 16, 0, 0);
}

__device__ __forceinline__ int swz(int row, int ch) { return row * ROWB + ((ch ^ ((row >> 1) & 7)) << 4); }

constexpr int GROUP_M = 8;   // row tiles per group of the tile order
constexpr int kCUs = 256;    // compute units of an MI355X

// instruction classes of __builtin_amdgcn_sched_group_barrier
constexpr int SG_MFMA = 0x008, SG_VMEM_READ = 0x020, SG_DS_READ = 0x100;

// Lane layout of the two matrix instructions (wave64).  Operands: lane l holds 8 consecutive k of
// row (l mod MI) of its 16 x 32 (MI 16) or 32 x 16 (MI 32) block, at k-chunk l / MI.  Result:
// element r of lane l is row 4 (l / 16) + r (MI 16) or out_row32(r, l) (MI 32), column l mod MI.
__device__ __forceinline__ int out_row32(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }
template <int MI>
__device__ __forceinline__ int in_chunk(int ks, int lane) {   // 16-byte chunk of a 128-byte row
  if constexpr (MI == 32)
    return 2 * ks + (lane >> 5);
  else
    return 4 * ks + (lane >> 4);
}
__device__ __forceinline__ f32x16 mfma_op(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_op(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// s_waitcnt vmcnt(N) lgkmcnt(0) for a compile-time N
template <int N>
__device__ __forceinline__ void wait_vm_lgkm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// ---------------------------------------------------------------------------
// The large bf16 products: BM x 256 tiles (BM 256, 192 or 128) on v_mfma_f32_16x16x32_bf16, eight
// waves, two per SIMD, each with two 16 HM-row by two 32-column blocks: rows from either half of
// the A tile, columns from either half of the B tile (the gate/up product: W_g, then W_u).
//   * A k-tile is four products of a half by a half.  Each half is read from LDS into registers
//     one product ahead, so a half of a stage is free again half a k-tile after its k-tile began,
//     and its loads for k-tile kt + 2 are issued then: they have one to one and a half k-tiles to
//     land (half a k-tile to one with whole stages), and the waits leave the loads of one k-tile in
//     flight (8, 7 and 6 a wave at 256, 192 and 128 rows).  Two barriers a k-tile.
//   * The loads write the LDS that the fragment reads read, so the compiler keeps their order:
//     they are written in the order they shall issue in, one between two MFMAs.  Issued as a burst
//     ahead of the reads (the order of the source before), the same loop lost all of its gain.
//   * The 16 x 16 x 32 instruction: at the same nominal rate as 32 x 32 x 16 it sustains a higher
//     clock on random data under the board's power limit.
// What bounds it: the matrix cores are busy for 75 % of its cycles (counters of the 8B stack's
// gate/up and down; the loop with whole stages 67 %), at the clock that the power limit leaves on
// random operands, 1.7-1.8 GHz.  A register-only loop of the same instruction has 91-94 % at 1.87 GHz
// (on zeros 96 % at 2.32).  The other quarter is waiting, at the two barriers and for loads and fragments (25 %
// of the waves' time); the fragment reads take 29 % of the LDS's cycles, bank conflicts 0.3 %.  4096 rows of the
// Llama-3.1-8B gate/up product: 1.84 PFLOP/s on zeros (whole stages 1.57), 1.44 on random operands
// (1.38); 20047 rows 3510 -> 3390 us, its down product 1845 -> 1760 us, 2995 rows on 192-row tiles
// 550 -> 525 and 265 -> 257 us.  Four waves of 128 x 128 (a third fewer LDS reads) reached 1.39.
// Epilogues: the gate/up products finish in registers and stage bf16; the others stage 16-row
// blocks in fp32 and take 8-column pieces (emit8) or the whole block (block).
// A grid with gridDim.y = S > 1 splits K as mfma_gemm does.
// ---------------------------------------------------------------------------

// An epilogue with a block() member takes each staged block of 16 rows whole, instead of 8-column
// row pieces through emit8().
template <class E, class = void>
struct BlockEpilogue : std::false_type {};
template <class E>
struct BlockEpilogue<E, std::void_t<decltype(&E::block)>> : std::true_type {};
// A two-product epilogue with kDualHook takes the accumulators of a finished wave tile itself (the
// backward of the gated SwiGLU) instead of the forward's SiLU(gate) * up staging.
template <class E, class = void>
struct DualHook : std::false_type {};
template <class E>
struct DualHook<E, std::void_t<decltype(E::kDualHook)>> : std::true_type {};

// An epilogue with kTwoTerm ends a product of two terms, A B^T + A2 B^T (ARows::base2)
template <class E, class = void>
struct TwoTerm : std::false_type {};
template <class E>
struct TwoTerm<E, std::void_t<decltype(E::kTwoTerm)>> : std::true_type {};

// An epilogue with kSixTerm ends a product of fp32 operands in three bf16 terms each, x = x0 + x1 + x2 with
// x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1): 24 bits, as fp32 has.  Of the nine products
// of terms the six of at least 2^-16 of the largest are formed, one after another along K; what is
// left out is 2^-24 of it, as an fp32 rounding is.  Six bf16 products run at 1.4 PFLOP/s / 6 = 230 TFLOP/s
// where the fp32 matrix cores peak at 157.
template <class E, class = void>
struct SixTerm : std::false_type {};
template <class E>
struct SixTerm<E, std::void_t<decltype(E::kSixTerm)>> : std::true_type {};
constexpr uint32_t kTermA = 0x120100, kTermB = 0x102010;   // term of the s-th product: bits 4 s

// An epilogue with kColumns prepares what its columns combine with once a tile (Epi::Cols, for the eight
// columns that a lane emits in every row block).
template <class E, class = void>
struct ColumnsHook : std::false_type {
  struct Cols {};
};
template <class E>
struct ColumnsHook<E, std::void_t<decltype(E::kColumns)>> : std::true_type {
  using Cols = typename E::Cols;
};
// An epilogue with kDeviceDepth knows K on the device: depth(), at most the host's
template <class E, class = void>
struct DeviceDepth : std::false_type {};
template <class E>
struct DeviceDepth<E, std::void_t<decltype(E::kDeviceDepth)>> : std::true_type {};

template <int BM_, bool DUAL_>
struct Phase {
  static constexpr int WN = 4, NW = 8, NT = 512;
  static constexpr int HB = 2;                  // 16-column fragments per wave and half
  static constexpr int BM = BM_, BN = 256;
  static constexpr bool DUAL = DUAL_;
  static constexpr int HM = BM / 64;            // 16-row fragments per wave and half
  static constexpr int STAGE = (BM + BN) * ROWB;
  static constexpr int OUT_N = DUAL ? 128 : 256;
  static constexpr int A_LD = BM / 8 / NW;      // 1 KiB stage loads per wave: A
  static constexpr int A1 = BM / 16 / NW;       // ... of the first half alone
  static constexpr int BH = 16 / NW;            // ... of half of B
  static constexpr int L1 = A1 + BH, L2 = A_LD - A1 + BH;
  static constexpr int SPLIT = A_LD % 2;        // loads of the second group that the first half needs too
  static constexpr int ON = 32;                 // output columns per wave and half
};

template <class C, class Epi>
__device__ __forceinline__ void swiglu_bwd_tile(const Epi& epi, f32x4 (&acc)[2 * C::HM][4], unsigned char* smem, int m0,
                                                int nt, int wave, int wm, int wn, int M, int lane);

template <class C, class Epi>
__device__ __forceinline__ void phase_tile(const ARows<bf16_t>& A, const BRows<bf16_t>& B, const Epi& epi, int M,
                                           int mt_act, int K, int n_tiles, unsigned char* smem, int tile, int slice,
                                           int slices) {
  constexpr int BM = C::BM, HM = C::HM, HB = C::HB, NW = C::NW, BH = C::BH;
  if (tile < 0 || tile >= mt_act * n_tiles) return;
  const int grp = tile / (GROUP_M * n_tiles), rem = tile % (GROUP_M * n_tiles);
  const int gsz = min(GROUP_M, mt_act - grp * GROUP_M);
  const int mt = grp * GROUP_M + rem % gsz, nt = rem / gsz;
  uint32_t turn = A.turn;
  if constexpr (DeviceDepth<Epi>::value) {
    K = epi.depth();
    turn = K / BK;
    if constexpr (SixTerm<Epi>::value) K *= 6;
  }
  // k / turn by a product (turn < 2^14, so exact for the 6 turn k-tiles there are)
  [[maybe_unused]] const uint32_t inv_turn = SixTerm<Epi>::value ? 0xffffffffu / turn + 1 : 0;
  const int m0 = mt * BM;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  const int rsub = lane >> 3;

  const unsigned char* a_base = reinterpret_cast<const unsigned char*>(A.base);
  uint32_t a_off[C::A_LD], b_off[2 * BH];
#pragma unroll
  for (int i = 0; i < C::A_LD; ++i) {
    const int r = 8 * (i * NW + wave) + rsub;
    const int ch = (lane & 7) ^ ((r >> 1) & 7);
    const int m = min(m0 + r, M - 1);
    const int row = A.idx ? A.idx[m] : m;
    a_off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(A.ld * 2) + ch * 16;
  }
  const unsigned char* b_base[2 * BH];
#pragma unroll
  for (int i = 0; i < 2 * BH; ++i) {
    const int blk = 8 * (i * NW + wave);   // first of eight rows, wave-uniform
    const int r = blk + rsub;
    const int ch = (lane & 7) ^ ((r >> 1) & 7);
    const bool second = C::DUAL ? blk >= 128 : nt * 256 + blk >= B.split;
    int row = min(C::DUAL ? nt * 128 + (r & 127) : nt * 256 + r - (second ? B.split : 0), B.last);
    if (B.idx) row = B.idx[row];
    b_base[i] = reinterpret_cast<const unsigned char*>(second ? B.b1 : B.b0);
    b_off[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(B.ld * 2) + ch * 16;
  }
  // split K: slice y of S covers k-tiles [y nkt / S, (y + 1) nkt / S), at least two
  const int nkt = K / BK;
  const int kt0 = slice * nkt / slices;
  const int nk = (slice + 1) * nkt / slices - kt0;
  const unsigned char* a_base2 = reinterpret_cast<const unsigned char*>(A.base2);
  // i-th load of the wave, k-tile kt of the slice
  auto at = [&](const unsigned char* base, const unsigned char* base2, size_t term, uint32_t terms, int k) {
    if constexpr (SixTerm<Epi>::value) {
      const uint32_t p = __umulhi(static_cast<uint32_t>(k), inv_turn);
      return base + (terms >> (4 * p) & 15u) * (term * 2) + (static_cast<uint32_t>(k) - p * turn) * ROWB;
    } else {
      const bool two = TwoTerm<Epi>::value && k >= A.turn;
      return (two ? base2 : base) + static_cast<uint32_t>(two ? k - A.turn : k) * ROWB;
    }
  };
  auto ldA = [&](int i, int kt) {
    load_lds16(at(a_base, a_base2, A.term, kTermA, kt0 + kt) + a_off[i],
               smem + (kt & 1) * C::STAGE + (i * NW + wave) * 1024);
  };
  auto ldB = [&](int i, int kt) {
    load_lds16(at(b_base[i], b_base[i], B.term, kTermB, kt0 + kt) + b_off[i],
               smem + (kt & 1) * C::STAGE + BM * ROWB + (i * NW + wave) * 1024);
  };
  // group 1: the first half of A and B; group 2: the rest (the piece of A that both halves share first)
  auto ld1 = [&](int i, int kt) { i < C::A1 ? ldA(i, kt) : ldB(i - C::A1, kt); };
  auto ld2 = [&](int i, int kt) {
    i < C::A_LD - C::A1 ? ldA(C::A1 + i, kt) : ldB(BH + i - (C::A_LD - C::A1), kt);
  };

  f32x4 acc[2 * HM][2 * HB];
#pragma unroll
  for (int a = 0; a < 2 * HM; ++a)
#pragma unroll
    for (int b = 0; b < 2 * HB; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int l15 = lane & 15;
  bf16x8 fa0[HM][2], fa1[HM][2], fb0[HB][2], fb1[HB][2];
  // fragment addresses: the chunk swizzle only depends on the lane (the blocks start at multiples of
  // 16 rows), so a fragment is a constant away from one of four addresses in the stage
  uint32_t offA[2], offB[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    offA[ks] = swz(wm * (BM / 4) + l15, in_chunk<16>(ks, lane));
    offB[ks] = BM * ROWB + swz(wn * 16 * HB + l15, in_chunk<16>(ks, lane));
  }
  auto rdA = [&](bf16x8 (&f)[HM][2], const unsigned char* st, int half, int i) {
    const int ks = i / HM, a = i % HM;
    f[a][ks] = *reinterpret_cast<const bf16x8*>(st + offA[ks] + (half * (BM / 2) + 16 * a) * ROWB);
  };
  auto rdB = [&](bf16x8 (&f)[HB][2], const unsigned char* st, int half, int i) {
    const int ks = i / HB, b = i % HB;
    f[b][ks] = *reinterpret_cast<const bf16x8*>(st + offB[ks] + (half * 128 + 16 * b) * ROWB);
  };
  auto mm = [&](const bf16x8 (&fa)[HM][2], const bf16x8 (&fb)[HB][2], int ha, int hb) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int a = 0; a < HM; ++a)
#pragma unroll
        for (int b = 0; b < HB; ++b)
          acc[ha * HM + a][hb * HB + b] = mfma_op(fa[a][ks], fb[b][ks], acc[ha * HM + a][hb * HB + b]);
  };
  // The memory operations of a phase in program order: a stage load after every EV-th fragment read (the
  // compiler keeps their order, as the loads write the LDS that the reads read), and the
  // schedule: one of them after each MFMA.
  auto mem = [&](auto nr_, auto nl_, auto ev_, auto rd, auto ld) {
    constexpr int nr = decltype(nr_)::value, nl = decltype(nl_)::value, ev = decltype(ev_)::value;
    int l = 0;
#pragma unroll
    for (int i = 0; i < nr; ++i) {
      rd(i);
      if (i % ev == ev - 1 && l < nl) ld(l++);
    }
#pragma unroll
    for (int i = 0; i < nl; ++i)
      if (i >= l) ld(i);
  };
  auto weave = [&](auto nm_, auto nr_, auto nl_, auto ev_) {
    constexpr int nm = decltype(nm_)::value, nl = decltype(nl_)::value, nr = decltype(nr_)::value,
                  ev = decltype(ev_)::value;
    int r = 0, l = 0;
#pragma unroll
    for (int i = 0; i < nm; ++i) {
      __builtin_amdgcn_sched_group_barrier(SG_MFMA, 1, 0);
      if (r < nr) {
        __builtin_amdgcn_sched_group_barrier(SG_DS_READ, 1, 0);
        ++r;
        if (r % ev == 0 && l < nl) {
          __builtin_amdgcn_sched_group_barrier(SG_VMEM_READ, 1, 0);
          ++l;
        }
      } else if (l < nl) {
        __builtin_amdgcn_sched_group_barrier(SG_VMEM_READ, 1, 0);
        ++l;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
#define IC(n) std::integral_constant<int, (n)>()
  constexpr int L1 = C::L1, L2 = C::L2, SP = C::SPLIT, NM = 2 * HM * HB;
  // MODE 2: tile kt + 2 is loaded; 1: the last but one; 0: the last
  auto ktile = [&](int kt, auto mode_) {
    constexpr int mode = decltype(mode_)::value;
    const unsigned char* st = smem + (kt & 1) * C::STAGE;
    const unsigned char* nx = smem + ((kt + 1) & 1) * C::STAGE;
    wait_vm_lgkm<mode == 0 ? 0 : L1 + L2>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    mem(IC(2 * HB + 2 * HM), IC(mode == 2 ? L1 : 0), IC(2),
        [&](int i) { i < 2 * HB ? rdB(fb1, st, 1, i) : rdA(fa1, st, 1, i - 2 * HB); }, [&](int i) { ld1(i, kt + 2); });
    mm(fa0, fb0, 0, 0);
    weave(IC(NM), IC(2 * HB + 2 * HM), IC(mode == 2 ? L1 : 0), IC(2));
    mm(fa0, fb1, 0, 1);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (mode != 0) {
      wait_vm_lgkm<(mode == 2 ? L1 + L2 : L2) - SP>();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      mem(IC(2 * HM), IC(mode == 2 ? L2 : 0), IC(1), [&](int i) { rdA(fa0, nx, 0, i); }, [&](int i) { ld2(i, kt + 2); });
    }
    mm(fa1, fb0, 1, 0);
    weave(IC(NM), IC(mode ? 2 * HM : 0), IC(mode == 2 ? L2 : 0), IC(1));
    if constexpr (mode != 0)
#pragma unroll
      for (int i = 0; i < 2 * HB; ++i) rdB(fb0, nx, 0, i);
    mm(fa1, fb1, 1, 1);
    weave(IC(NM), IC(mode ? 2 * HB : 0), IC(0), IC(1));
  };
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int i = 0; i < L1; ++i) ld1(i, t);
#pragma unroll
    for (int i = 0; i < L2; ++i) ld2(i, t);
  }
  wait_vm_lgkm<L1 + 2 * L2 - SP>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < 2 * HM; ++i) rdA(fa0, smem, 0, i);
#pragma unroll
  for (int i = 0; i < 2 * HB; ++i) rdB(fb0, smem, 0, i);
  int kt = 0;
  for (; kt + 2 < nk; ++kt) ktile(kt, IC(2));
  ktile(kt, IC(1));
  ktile(kt + 1, IC(0));
#undef IC
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();

  if constexpr (DualHook<Epi>::value) {
    swiglu_bwd_tile<C>(epi, acc, smem, m0, nt, wave, wm, wn, M, lane);
  } else if constexpr (C::DUAL) {
    // rows of half h: m0 + h BM/2 + wm BM/4 + ..; the wave's 32 columns of act, gate in acc[.][0..1], up in [2..3]
    constexpr int ON = 16 * HB, SP2 = ON + 8, CPR = ON / 8;
    bf16_t* stg = reinterpret_cast<bf16_t*>(smem) + wave * (32 * HM * SP2);
#pragma unroll
    for (int a = 0; a < 2 * HM; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int b = 0; b < HB; ++b) {
          const float g = acc[a][b][r], u = acc[a][HB + b][r];
          stg[(16 * a + 4 * (lane >> 4) + r) * SP2 + 16 * b + l15] =
              f32_to_bf16(g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u);
        }
#pragma unroll
    for (int p = 0; p < 2 * HM * 16 * CPR / kWave; ++p) {
      const int e = lane + kWave * p, i = e / CPR, c8 = (e % CPR) * 8;
      const int h = i / (16 * HM), m = m0 + h * (BM / 2) + wm * (BM / 4) + i - h * 16 * HM;
      const u32x4 v = *reinterpret_cast<const u32x4*>(stg + i * SP2 + c8);
      if (m < M) epi.emit_packed(m, nt * 128 + wn * ON + c8, v);
    }
  } else {
    // per half of B: 32 columns; 16-row blocks staged as fp32
    constexpr int ON = 16 * HB, OP = 2 * ON + 4, CPR = ON / 4, PP = 16 * CPR / kWave;
    float* stg = reinterpret_cast<float*>(smem) + wave * (16 * OP);
    typename Epi::Pre pre[2 * HM][PP];
    // rows of fragment a, columns of the staged pair of 32-column blocks
    auto row_of = [&](int a, int i) { return m0 + (a / HM) * (BM / 2) + wm * (BM / 4) + 16 * (a % HM) + i; };
    auto col_of = [&](int c8) { return nt * 256 + (c8 / ON) * 128 + wn * ON + c8 % ON; };
    auto fetch = [&](int a) {
#pragma unroll
      for (int p = 0; p < PP; ++p) {
        const int e = lane + kWave * p;
        pre[a][p] = epi.prep(min(row_of(a, e / CPR), M - 1), col_of((e % CPR) * 8));
      }
    };
    typename ColumnsHook<Epi>::Cols cols;
    if constexpr (ColumnsHook<Epi>::value) cols = epi.cols(col_of((lane % CPR) * 8));   // CPR divides the wave
    // what the epilogue combines with (hbar rows) is fetched some fragments ahead of the staging
    constexpr int AHEAD = TwoTerm<Epi>::value ? 2 : 4;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(a);
#pragma unroll
    for (int a = 0; a < 2 * HM; ++a) {
      if (a + AHEAD < 2 * HM) fetch(a + AHEAD);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int b = 0; b < 2 * HB; ++b) stg[(4 * (lane >> 4) + r) * OP + 16 * b + l15] = acc[a][b][r];
      if constexpr (BlockEpilogue<Epi>::value) {
        epi.block(stg, OP, ON, row_of(a, 0), col_of(0), M, lane);
        epi.block(stg + ON, OP, ON, row_of(a, 0), col_of(ON), M, lane);
      } else {
#pragma unroll
        for (int p = 0; p < PP; ++p) {
          const int e = lane + kWave * p, i = e / CPR, c8 = (e % CPR) * 8;
          const int m = row_of(a, i);
          if constexpr (ColumnsHook<Epi>::value) {
            if (m < M) epi.emit8(cols, m, col_of(c8), stg + i * OP + c8);
          } else {
            if (m < M) epi.emit8(pre[a][p], m, col_of(c8), stg + i * OP + c8);
          }
        }
      }
    }
  }
}


// Row tiles of M rows, at most those the grid was sized for
__device__ __forceinline__ int row_tiles(int M, int M_max, int BM) {
  return min((M_max + BM - 1) / BM, (M + BM - 1) / BM);
}
// The tile of workgroup b: each XCD (b mod 8) takes a contiguous range of the grouped order; -1: none
__device__ __forceinline__ int tile_of(int b, int tiles) {
  const int per = (tiles + 7) >> 3;
  return (b >> 3) < per ? (b & 7) * per + (b >> 3) : -1;
}

template <class C, class Epi>
__global__ __launch_bounds__(512, 2) void phase_gemm(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi,
                                                     const int* __restrict__ m_count, int M_max, int K, int n_tiles) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * C::STAGE];
  const int M = m_count ? *m_count : M_max, mt = row_tiles(M, M_max, C::BM);
  phase_tile<C>(A, B, epi, M, mt, K, n_tiles, smem, tile_of(blockIdx.x, mt * n_tiles), blockIdx.y, gridDim.y);
}

// Tile height for M rows: the launch's time in rounds of workgroups over the CUs, times the
// relative duration of a round (measured on the Llama-3.1-8B gate/up and down shapes at 0.4k to 20k
// rows: 54-57, 78 and 97 us for 128-, 192- and 256-row tiles at K = 4096; 187, 258 and 345 at
// 14336).  The smaller tiles move more bytes per product and only pay while their finer rounds
// leave fewer CUs idle, so beyond four (128) and eight (192) rounds they are not considered.
// SPILL: the epilogues of the two backwards, whose 256-row tiles spill 96 and 36 registers and so are
// hardly faster a row than 192-row ones.  With the weights above against these, whole calls at the 8B shape:
// block backward 1135 -> 1085 us at 2800 tokens, 5768 -> 5511 at 16000, router backward 1010 -> 962 at
// 8192; 256 rows stay where they make a single round (block backward of 700 tokens: 626, on 128 rows 636).
template <bool SPILL>
__host__ __device__ inline int phase_rows(int M, int n_tiles) {
  auto tiles = [&](int BM) { return (M + BM - 1) / BM * n_tiles; };
  auto cost = [&](int BM, int w) { return (tiles(BM) + kCUs - 1) / kCUs * w; };
  int best = 256, c = cost(256, SPILL ? 152 : 125);
  if ((SPILL || tiles(192) <= 8 * kCUs) && cost(192, 100) < c) {
    best = 192;
    c = cost(192, 100);
  }
  if (tiles(128) <= 4 * kCUs && cost(128, SPILL ? 80 : 75) < c) best = 128;
  return best;
}
template <class Epi>
constexpr bool kSpill = DualHook<Epi>::value || TwoTerm<Epi>::value;

// one of the three tile heights, chosen on the device
template <bool DUAL, class Epi>
__device__ __forceinline__ void phase_any(int bm, const ARows<bf16_t>& A, const BRows<bf16_t>& B, const Epi& epi, int M,
                                          int mt, int K, int n_tiles, unsigned char* smem, int tile, int slice, int slices) {
  if (bm == 256)
    phase_tile<Phase<256, DUAL>>(A, B, epi, M, mt, K, n_tiles, smem, tile, slice, slices);
  else if (bm == 192)
    phase_tile<Phase<192, DUAL>>(A, B, epi, M, mt, K, n_tiles, smem, tile, slice, slices);
  else
    phase_tile<Phase<128, DUAL>>(A, B, epi, M, mt, K, n_tiles, smem, tile, slice, slices);
}

// Threshold routing: the host only knows an upper bound of the row count, so the workgroups choose
// the tile height themselves from the count on the device.
template <bool DUAL, class Epi>
__global__ __launch_bounds__(512, 2) void phase_gemm_any(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi,
                                                         const int* __restrict__ m_count, int M_max, int K,
                                                         int n_tiles) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * Phase<256, DUAL>::STAGE];
  const int M = min(*m_count, M_max);
  const int bm = phase_rows<kSpill<Epi>>(M, n_tiles), mt = row_tiles(M, M_max, bm);
  phase_any<DUAL>(bm, A, B, epi, M, mt, K, n_tiles, smem, tile_of(blockIdx.x, mt * n_tiles), blockIdx.y, gridDim.y);
}

// exact: M_max is the row count (m_count, if given, holds at most that)
template <bool DUAL, class Epi>
hipError_t run_phase(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi, const int* m_count, int M_max, int N_out, int K,
                     hipStream_t s, bool exact = true) {
  const int n_tiles = N_out / Phase<256, DUAL>::OUT_N;
  if (M_max <= 0 || n_tiles <= 0) return hipSuccess;
  const auto blocks = [&](int BM) { return ((M_max + BM - 1) / BM * n_tiles + 7) / 8 * 8; };
  if constexpr (!TwoTerm<Epi>::value) {   // the products of two terms know their rows
    if (!exact && m_count) {
      // enough for any choice at any count up to M_max
      const int grid = std::max({blocks(256), kSpill<Epi> ? blocks(192) : std::min(blocks(192), 8 * kCUs),
                                 std::min(blocks(128), 4 * kCUs)});
      phase_gemm_any<DUAL, Epi><<<grid, 512, 0, s>>>(A, B, epi, m_count, M_max, K, n_tiles);
      return hipGetLastError();
    }
  }
  switch (phase_rows<kSpill<Epi>>(M_max, n_tiles)) {
    case 256: phase_gemm<Phase<256, DUAL>, Epi><<<blocks(256), 512, 0, s>>>(A, B, epi, m_count, M_max, K, n_tiles); break;
    case 192: phase_gemm<Phase<192, DUAL>, Epi><<<blocks(192), 512, 0, s>>>(A, B, epi, m_count, M_max, K, n_tiles); break;
    default: phase_gemm<Phase<128, DUAL>, Epi><<<blocks(128), 512, 0, s>>>(A, B, epi, m_count, M_max, K, n_tiles); break;
  }
  return hipGetLastError();
}

// K split S ways over 128-row tiles, for products of too few tiles to fill the CUs
template <class Epi>
hipError_t run_phase_split(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi, const int* m_count, int M_max, int N_out, int K,
                           int S, hipStream_t s) {
  using C = Phase<128, false>;
  const int n_tiles = N_out / C::OUT_N;
  const dim3 grid(((M_max + 127) / 128 * n_tiles + 7) / 8 * 8, S);
  phase_gemm<C, Epi><<<grid, 512, 0, s>>>(A, B, epi, m_count, M_max, K, n_tiles);
  return hipGetLastError();
}

}  // namespace
}  // namespace hero
