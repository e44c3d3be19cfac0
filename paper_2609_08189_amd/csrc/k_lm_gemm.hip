// The products of the language-model loss over one piece of the vocabulary (k_lm_loss.hip has the formulas):
//   logits   l = x[idx] W^T        -> e = exp(l - ref) as stored, and its sums a row and 64 columns; few
//                                     tiles: K slices of l in fp32, which the combining pass turns into e
//   dx       acc (+)= e W          B = W^T [d][pitch of the vocabulary]
//   dW       g = (p - [target])^T  = W x^T with an epilogue, the tokens contiguous
//            dW = unit g x         B = x^T [d][tokens]
// All on the phase-ordered core, whose rate on random operands (1.3 to 1.45 PFLOP/s) bounds them.  fp32 models: the
// same products on three-term operands (kLmSplit).
#include "hero_gemm.h"

#include "hero_kernels.h"

namespace hero {
namespace {

// Where a logit may stand above its row's reference before the piece takes one of its own: e stays far
// from the end of the range (e^60 summed over any vocabulary, times any weight, is below 2^120).
constexpr float kLmAbove = 60.0f;

template <bool SIX>
struct Six {};
template <>
struct Six<true> {
  static constexpr bool kSixTerm = true;
};

// eight values as stored: bf16, or three bf16 terms `term` elements apart
template <bool SIX>
__device__ __forceinline__ void st8_terms(bf16_t* p, size_t term, const float* v) {
  if constexpr (!SIX) {
    st8(p, v);
  } else {
    float r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = v[k];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      st8(p + t * term, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] -= bf16_to_f32(f32_to_bf16(r[k]));
    }
  }
}

template <bool SIX>
__device__ __forceinline__ float lm_exp(float x) {
  return SIX ? expf(x) : __expf(x);
}

// e[m][n] = exp(l - ref_m) for every column but the target's, whose share is kept apart (1 - p of a sure
// token would cancel in it).  ref is the target's logit, or what the row's earlier pieces raised it to, so
// no pass for a maximum is needed: e is a floating number whatever its size.  Where a logit is more than
// kLmAbove over it, the wave's 64 columns of that row take their own maximum as reference, and the pass
// over the partial sums brings them together.  The 64 columns of a row sit in eight neighbouring lanes.
template <bool STORE, bool SIX>
struct EpiLmExp : Six<SIX> {
  const float* ref;
  const int* tgt;
  int v0, cols, pitch;
  bf16_t* e;
  size_t term;
  float2* part;
  int parts;
  struct Pre {
    float ref;
    int tgt;
  };
  __device__ __forceinline__ Pre prep(int m, int) const { return {ref[m], tgt[m] - v0}; }
  __device__ __forceinline__ void emit8(const Pre& p, int m, int n, const float* v) const {
    float x[8], s = 0.f;
    float mx = v[0];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = v[k];
      mx = fmaxf(mx, x[k]);
    }
    float r = p.ref;
    // all lanes inside the vocabulary, away from their targets and their references good: the plain case
    const bool plain = n + 8 <= cols && static_cast<unsigned>(p.tgt - n) >= 8u && !(mx - r > kLmAbove);
    if (__all(plain)) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = lm_exp<SIX>(x[k] - r);
        s += x[k];
      }
    } else {
      mx = r;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (n + k < cols) mx = fmaxf(mx, x[k]);
      mx = fmaxf(mx, __shfl_xor(mx, 1, 8));
      mx = fmaxf(mx, __shfl_xor(mx, 2, 8));
      mx = fmaxf(mx, __shfl_xor(mx, 4, 8));
      if (mx - r > kLmAbove) r = mx;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[k] = n + k < cols && n + k != p.tgt ? lm_exp<SIX>(x[k] - r) : 0.f;
        s += x[k];
      }
    }
    if constexpr (STORE) {
      if (n < pitch) st8_terms<SIX>(e + static_cast<size_t>(m) * pitch + n, term, x);
    }
    s = group_sum<8>(s);
    if ((threadIdx.x & 7) == 0) part[static_cast<size_t>(m) * parts + (n >> 8) * 4 + ((n & 127) >> 5)] = {r, s};
  }
};

template <bool SIX>
struct EpiLmLogits : EpiStoreF32, Six<SIX> {};

// acc[m][n] = the piece's product, or alpha_m acc[m][n] + it
template <bool FIRST, bool SIX>
struct EpiLmAcc : Six<SIX> {
  float* out;
  int ld;
  const float* alpha;
  struct Pre {
    f32x4 o[FIRST ? 1 : 2];
    float a;
  };
  __device__ __forceinline__ float* at(int m, int n) const { return out + static_cast<size_t>(m) * ld + n; }
  __device__ __forceinline__ Pre prep(int m, int n) const {
    Pre p{};
    if constexpr (!FIRST) {
      p.o[0] = *reinterpret_cast<const f32x4*>(at(m, n));
      p.o[1] = *reinterpret_cast<const f32x4*>(at(m, n) + 4);
      p.a = alpha[m];
    }
    return p;
  }
  __device__ __forceinline__ void emit8(const Pre& p, int m, int n, const float* v) const {
    f32x4 lo = *reinterpret_cast<const f32x4*>(v), hi = *reinterpret_cast<const f32x4*>(v + 4);
    if constexpr (!FIRST) {
      lo += p.a * p.o[0];
      hi += p.a * p.o[1];
    }
    *reinterpret_cast<f32x4*>(at(m, n)) = lo;
    *reinterpret_cast<f32x4*>(at(m, n) + 4) = hi;
  }
};

// columns of the tokens that a product over them as K runs through: at least two k-tiles
__device__ __forceinline__ int lm_depth(const int* count) { return max(2 * BK, (*count + BK - 1) / BK * BK); }

// g[v][t] = p_tv - [v = target of t] for the counted rows t, zero behind them (the unit, scale / N, is
// dW's epilogue's); columns: the tokens' log sums and targets
template <bool SIX>
struct EpiLmG : Six<SIX> {
  static constexpr bool kColumns = true;
  const float *lse, *own;    // [rows] log sum of a row, p - 1 of its target
  const int *tgt, *count;
  int v0, pitch;
  bf16_t* g;
  size_t term;
  struct Cols {
    float lse[8];
    int tgt[8];
  };
  struct Pre {};
  __device__ __forceinline__ Pre prep(int, int) const { return {}; }
  __device__ __forceinline__ Cols cols(int n) const {
    Cols c;
    const int N = *count;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool in = n + k < N;
      c.lse[k] = in ? lse[n + k] : 0.f;
      c.tgt[k] = in ? tgt[n + k] - v0 : INT_MIN;
    }
    return c;
  }
  __device__ __forceinline__ void emit8(const Cols& c, int m, int n, const float* v) const {
    if (n >= pitch) return;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = c.tgt[k] == INT_MIN ? 0.f : lm_exp<SIX>(v[k] - c.lse[k]);
      if (c.tgt[k] == m) x[k] = own[n + k];
    }
    st8_terms<SIX>(g + static_cast<size_t>(m) * pitch + n, term, x);
  }
};

template <typename T, bool SIX>
struct EpiLmDw : Six<SIX> {   // dw[m][n] = unit acc, the tokens as K
  static constexpr bool kDeviceDepth = true;
  T* out;
  int ld;
  const int* count;
  float scale;
  bool mean;
  struct Pre {
    float c;
  };
  __device__ __forceinline__ int depth() const { return lm_depth(count); }
  __device__ __forceinline__ Pre prep(int, int) const { return {mean ? scale / static_cast<float>(max(*count, 1)) : scale}; }
  __device__ __forceinline__ void emit8(const Pre& p, int m, int n, const float* v) const {
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = p.c * v[k];
    st8(out + static_cast<size_t>(m) * ld + n, x);
  }
};

// The dx product on the tile height and K slices that the rows' plan names; slice z into acc + z M d.  Workgroups
// go to the XCDs round-robin: an XCD keeps to one slice (S < 8: 8 / S XCDs share one; S a multiple of 8: S / 8
// slices one after another), so that what its tiles read, all rows of e and of W^T over the slice's columns,
// passes through its L2 once.  With every slice spread over all XCDs, 1173 rows of d = 1024 against 50257 columns
// in 12 slices took 212 us (about 1 GB fetched where the operands are 220 MB).
template <class Epi>
__global__ __launch_bounds__(512, 2) void lm_dx_kernel(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi,
                                                       const int* __restrict__ m_count, const int* __restrict__ plan,
                                                       int M_max, int K, int n_tiles) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * Phase<256, false>::STAGE];
  const int M = min(*m_count, M_max), bm = *plan & 0xffff, S = *plan >> 16;
  const int mt = row_tiles(M, M_max, bm), tiles = mt * n_tiles;
  if (tiles == 0) return;
  const int x = static_cast<int>(blockIdx.x) & 7, q = static_cast<int>(blockIdx.x) >> 3;
  int z, tile;
  if (S >= 8) {
    z = x + 8 * (q / tiles);
    tile = q % tiles;
  } else {
    const int g = 8 / S, per = (tiles + g - 1) / g;
    z = x / g;
    tile = q < per ? x % g * per + q : -1;
  }
  if (z >= S) return;
  epi.out += static_cast<size_t>(z) * M * epi.ld;
  phase_any<false>(bm, A, B, epi, M, mt, K, n_tiles, smem, tile, z, S);
}

// g's product: as many columns as there are counted tokens, so the tile height is chosen on the device
template <class Epi>
__global__ __launch_bounds__(512, 2) void lm_g_product(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi, int M, int K) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * Phase<256, false>::STAGE];
  const int n_tiles = (lm_depth(epi.count) + 255) / 256;
  const int bm = phase_rows<false>(M, n_tiles), mt = row_tiles(M, M, bm);
  phase_any<false>(bm, A, B, epi, M, mt, K, n_tiles, smem, tile_of(blockIdx.x, mt * n_tiles), 0, 1);
}

// The dW product in K slices, for heads of few tiles: slice z into part + z M d
template <bool SIX>
struct EpiLmDwPart : EpiLmAcc<true, SIX> {
  static constexpr bool kDeviceDepth = true;
  const int* count;
  __device__ __forceinline__ int depth() const { return lm_depth(count); }
};
template <class Epi>
__global__ __launch_bounds__(512, 2) void lm_dw_part_kernel(ARows<bf16_t> A, BRows<bf16_t> B, Epi epi, int M, int n_tiles,
                                                            int slices) {
  using C = Phase<128, false>;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * C::STAGE];
  const int S = lm_dw_slices_of(slices, epi.depth()), z = blockIdx.y, mt = row_tiles(M, M, C::BM);
  if (z >= S) return;
  epi.out += static_cast<size_t>(z) * M * epi.ld;
  phase_tile<C>(A, B, epi, M, mt, 0, n_tiles, smem, tile_of(blockIdx.x, mt * n_tiles), z, S);
}

// dW of few rows: little to compute and all of dW to write.  A workgroup takes 128 head rows, a wave 32 of them
// (operand B: their g, held; bf16: two terms of it), and `width` columns of d (A: rows of x^T, staged in LDS, so that
// no load waits behind a store: with both in one loop 26 rows of d = 3584 against 116669 took 303 us, so 162, 5.2 TB/s).
// Rows of A are dealt out so that a lane's sixteen results are neighbours, and the four lanes of a head row write 64
// elements of it in whole lines.  G: groups of 32 (bf16) or 16 (fp32) tokens.
template <typename T, int G>
__device__ __forceinline__ void dw_few(const LmRows& a, int cols, const T* __restrict__ g, const T* __restrict__ xT, int pitch,
                                       int width, T* __restrict__ dw, unsigned char* xs) {
  constexpr bool F32 = std::is_same_v<T, float>;
  typedef std::conditional_t<F32, f32x4, bf16x8> Frag;
  constexpr int E = F32 ? 4 : 8, ROW = 64 * G + 16;   // bytes of a staged row: 16-byte reads of 16 rows miss each other
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, q = lane >> 4;
  const int i0 = blockIdx.y * width, di = min(width, a.d - i0);
  for (int e = threadIdx.x; e < di * 4 * G; e += 256)
    *reinterpret_cast<u32x4*>(xs + (e / (4 * G)) * ROW + e % (4 * G) * 16) = *reinterpret_cast<const u32x4*>(
        reinterpret_cast<const unsigned char*>(xT + static_cast<size_t>(i0 + e / (4 * G)) * pitch) + e % (4 * G) * 16);
  const float unit = F32 ? 1.0f : a.mean ? a.scale / static_cast<float>(max(a.counts[0], 1)) : a.scale;
  constexpr int TERMS = F32 ? 1 : 2;   // of g
  Frag fg[2][G][TERMS];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int k = 0; k < G; ++k)
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
        fg[b][k][t] = *reinterpret_cast<const Frag*>(
            g + (static_cast<size_t>(t) * cols + min(static_cast<int>(blockIdx.x) * 128 + wave * 32 + 16 * b + l15, cols - 1)) * pitch +
            (4 * k + q) * E);
  __syncthreads();
  for (int i = 0; i < di; i += 64) {
    f32x4 acc[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      const unsigned char* row = xs + (i + 16 * (l15 >> 2) + 4 * j + (l15 & 3)) * ROW;
#pragma unroll
      for (int k = 0; k < G; ++k) {
        const Frag fx = *reinterpret_cast<const Frag*>(row + (4 * k + q) * 16);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fx[e], fg[b][k][0][e], acc[b][j], 0, 0, 0);
          } else {
            acc[b][j] = mfma_op(fx, fg[b][k][1], acc[b][j]);
            acc[b][j] = mfma_op(fx, fg[b][k][0], acc[b][j]);
          }
        }
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int n = blockIdx.x * 128 + wave * 32 + 16 * b + l15;
      if (n >= cols) continue;
      T* out = dw + static_cast<size_t>(n) * a.d + i0 + i + 16 * q;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = unit * acc[b][2 * h + (k >> 2)][k & 3];
        st8(out + 8 * h, v);
      }
    }
  }
}

// as many groups as the counted tokens fill, of the MOST that the call may have
template <typename T, int MOST>
__global__ __launch_bounds__(256) void lm_dw_few(LmRows a, int cols, const T* __restrict__ g, const T* __restrict__ xT,
                                                 int pitch, int width, T* __restrict__ dw) {
  constexpr int GROUP = std::is_same_v<T, float> ? 16 : 32;
  __shared__ __attribute__((aligned(16))) unsigned char xs[(MOST <= 4 ? 256 : 128) * (64 * MOST + 16)];
  const int N = a.counts[0];
  if (MOST == 1 || N <= GROUP) return dw_few<T, 1>(a, cols, g, xT, pitch, width, dw, xs);
  if constexpr (MOST >= 2)
    if (MOST == 2 || N <= 2 * GROUP) return dw_few<T, 2>(a, cols, g, xT, pitch, width, dw, xs);
  if constexpr (MOST >= 4)
    if (MOST == 4 || N <= 4 * GROUP) return dw_few<T, 4>(a, cols, g, xT, pitch, width, dw, xs);
  if constexpr (MOST >= 8) dw_few<T, 8>(a, cols, g, xT, pitch, width, dw, xs);
}

// ---------------------------------------------------------------------------
// Logits of few rows: the head streams past all of them at once.  A workgroup takes 128 head rows and every row of
// x (up to 16 TB), a ring of NS k-tiles in LDS, NS - 1 of them in flight, so that two workgroups a CU keep some 100 KB
// under way: on the large products' tiles, of which small heads have too few, two k-tiles of 125 CUs drew 2.9 TB/s.
// Operand A: 32 head rows a wave, B: the rows of x.  One barrier a k-tile: past it every wave has the tile's loads of
// all waves, and none reads the tile before any more, whose place the next loads take.
// fp32: a k-tile's 128 bytes of a row are 32 elements, and a lane's 16 bytes feed four matrix instructions.
// ---------------------------------------------------------------------------
template <typename T, int TB, int NS>
struct FewRing {
  static constexpr bool F32 = std::is_same_v<T, float>;
  static constexpr int BV = 128, BX = 16 * TB, STAGE = (BV + BX) * ROWB;
  static constexpr int XL = TB < 4 ? 1 : TB / 2;   // loads a wave of x (TB 1: two waves repeat the others')
  static constexpr int L = 4 + XL;
  typedef std::conditional_t<F32, f32x4, bf16x8> Frag;
  // acc[f][b]: rows 16 f of the wave's 32 of w (`rows` of them, the last repeated), rows 16 b of x; w and x at k-tile 0 of
  // nkt >= NS - 1, x_row(r) the byte offset of row r
  template <class X>
  static __device__ __forceinline__ void run(const unsigned char* w, size_t w_bytes, int rows, const unsigned char* x, X x_row,
                                             int nkt, unsigned char* smem, f32x4 (&acc)[2][TB]) {
    const int lane = threadIdx.x & 63, l15 = lane & 15, rsub = lane >> 3;
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    uint32_t w_off[4], x_off[XL];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 8 * (4 * i + wave) + rsub, ch = (lane & 7) ^ ((r >> 1) & 7);
      w_off[i] = static_cast<uint32_t>(min(r, rows - 1)) * static_cast<uint32_t>(w_bytes) + ch * 16;
    }
    const auto x_block = [&](int i) { return (4 * i + wave) % (2 * TB); };   // of eight rows
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const int r = 8 * x_block(i) + rsub, ch = (lane & 7) ^ ((r >> 1) & 7);
      x_off[i] = x_row(r) + ch * 16;
    }
    auto issue = [&](int kt) {
      unsigned char* st = smem + kt % NS * STAGE;
      const uint32_t kb = static_cast<uint32_t>(kt) * ROWB;
#pragma unroll
      for (int i = 0; i < 4; ++i) load_lds16(w + kb + w_off[i], st + (4 * i + wave) * 1024);
#pragma unroll
      for (int i = 0; i < XL; ++i) load_lds16(x + kb + x_off[i], st + BV * ROWB + x_block(i) * 1024);
    };
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NS - 1; ++k) issue(k);
    for (int kt = 0; kt < nkt; ++kt) {
      // this wave's loads of tile kt have landed (NS - 2 tiles behind it may be in flight; near the end all have)
      if (kt + NS - 1 <= nkt)
        wait_vm_lgkm<(NS - 2) * L>();
      else
        wait_vm_lgkm<0>();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if (kt + NS - 1 < nkt) issue(kt + NS - 1);
      const unsigned char* st = smem + kt % NS * STAGE;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int c = in_chunk<16>(ks, lane);
        Frag fw[2], fx[TB];
#pragma unroll
        for (int f = 0; f < 2; ++f) fw[f] = *reinterpret_cast<const Frag*>(st + swz(wave * 32 + 16 * f + l15, c));
#pragma unroll
        for (int b = 0; b < TB; ++b) fx[b] = *reinterpret_cast<const Frag*>(st + BV * ROWB + swz(16 * b + l15, c));
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
              for (int b = 0; b < TB; ++b)
                acc[f][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[f][e], fx[b][e], acc[f][b], 0, 0, 0);
        } else {
#pragma unroll
          for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int b = 0; b < TB; ++b) acc[f][b] = mfma_op(fw[f], fx[b], acc[f][b]);
        }
      }
    }
  }
};

// SCORE: no exponential is kept, so a part may take its own maximum as reference, and neither the rows nor their targets'
// logits are needed before: all tokens are rows (the head's passage costs the same), and one launch less comes first.
template <typename T, int TB, int NS, bool STORE, bool SCORE>
__device__ __forceinline__ void few_logits(const LmRows& a, const LmPiece& p, int M, unsigned char* smem) {
  typedef FewRing<T, TB, NS> R;
  constexpr bool F32 = R::F32;
  constexpr int BX = R::BX;
  const int lane = threadIdx.x & 63, l15 = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int v0 = blockIdx.x * R::BV;
  const size_t row_bytes = static_cast<size_t>(a.d) * sizeof(T);
  f32x4 acc[2][TB];
  R::run(static_cast<const unsigned char*>(a.w) + static_cast<size_t>(p.v0 + v0) * row_bytes, row_bytes, p.cols - v0,
         static_cast<const unsigned char*>(a.x),
         [&](int r) {
           const int m = min(r, M - 1);
           return static_cast<uint32_t>(SCORE ? m : a.idx[p.m0 + m]) * static_cast<uint32_t>(row_bytes);
         },
         static_cast<int>(row_bytes / ROWB), smem, acc);   // d >= 256, fp32 128: four k-tiles at least
  static_assert(NS <= 5, "the first loads are of tiles that exist");
  // every wave is past its last reads; the ring's memory holds the columns' maxima and sums now
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();
  float* top = reinterpret_cast<float*>(smem);     // [4][BX]
  float* sums = top + 4 * BX;
  const int n0 = v0 + wave * 32 + 4 * q;           // lane: columns n0 + 16 f + r of row 16 b + l15
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    float mx = -INFINITY;
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n0 + 16 * f + r < p.cols) mx = fmaxf(mx, acc[f][b][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    if (q == 0) top[wave * BX + 16 * b + l15] = mx;
  }
  __syncthreads();
  float ref[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int m = 16 * b + l15, mc = p.m0 + min(m, M - 1);
    const float t = fmaxf(fmaxf(top[m], top[BX + m]), fmaxf(top[2 * BX + m], top[3 * BX + m]));
    if constexpr (SCORE) {
      ref[b] = t == -INFINITY ? 0.f : t;
    } else {
      const float r0 = a.ref[mc];
      ref[b] = t - r0 > kLmAbove ? t : r0;
    }
    // of a token that does not count any value: its sums are not read
    const int tgt = SCORE ? static_cast<int>(static_cast<unsigned>(a.targets[mc]) - static_cast<unsigned>(n0)) : a.tgt[mc] - p.v0 - n0;
    float s = 0.f;
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      float o[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int k = 16 * f + r;
        o[r] = n0 + k < p.cols && k != tgt ? lm_exp<F32>(acc[f][b][r] - ref[b]) : 0.f;
        s += o[r];
      }
      if constexpr (STORE)
        if (m < M && n0 + 16 * f < p.pitch) {
          T* e = static_cast<T*>(p.e) + static_cast<size_t>(m) * p.pitch + n0 + 16 * f;
          if constexpr (F32)
            *reinterpret_cast<f32x4*>(e) = f32x4{o[0], o[1], o[2], o[3]};
          else
            *reinterpret_cast<uint2*>(e) = uint2{f32_to_bf16(o[0]) | static_cast<uint32_t>(f32_to_bf16(o[1])) << 16,
                                                 f32_to_bf16(o[2]) | static_cast<uint32_t>(f32_to_bf16(o[3])) << 16};
        }
    }
    s += __shfl_xor(s, 16, kWave);
    s += __shfl_xor(s, 32, kWave);
    if (q == 0) sums[wave * BX + m] = s;
  }
  __syncthreads();
  if (wave == 0 && q == 0)
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const int m = 16 * b + l15;
      if (m < M)
        p.part[static_cast<size_t>(m) * p.parts + blockIdx.x] = {
            ref[b], (sums[m] + sums[BX + m]) + (sums[2 * BX + m] + sums[3 * BX + m])};
    }
}

// The ring's width by the rows that count, up to MOST blocks of 16 (the host's bound, which sizes the LDS): fp32 products of
// all rows where 29 of 96 count: 894 us a call with both gradients, d = 2304 against 45397 columns, so 565.
template <int MOST>
constexpr int kFewBytes = MOST == 1 ? 4 * 144 * ROWB : MOST <= 4 ? 4 * 160 * ROWB : 3 * (128 + 16 * MOST) * ROWB;
template <int N>
using Int = std::integral_constant<int, N>;
template <int MOST, class F>
__device__ __forceinline__ void few_case(int M, F f) {
  if (MOST == 1 || M <= 16) return f(Int<1>(), Int<4>());
  if constexpr (MOST >= 2)
    if (MOST == 2 || M <= 32) return f(Int<2>(), Int<4>());
  if constexpr (MOST >= 4)
    if (MOST == 4 || M <= 64) return f(Int<4>(), Int<3>());
  if constexpr (MOST >= 6)
    if (MOST == 6 || M <= 96) return f(Int<6>(), Int<3>());
  if constexpr (MOST >= 8) f(Int<8>(), Int<3>());
}

template <typename T, int MOST, bool STORE, bool SCORE = false>
__global__ __launch_bounds__(256) void lm_logits_few(LmRows a, LmPiece p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kFewBytes<MOST>];
  const int M = SCORE ? a.T : *p.count;
  if (M == 0) return;
  if (SCORE && blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
  few_case<MOST>(M, [&](auto tb, auto ns) { few_logits<T, decltype(tb)::value, decltype(ns)::value, STORE, SCORE>(a, p, M, smem); });
}

// dx of few fp32 rows the same way: W^T streams past the rows of e, slice z of K into acc + z M d
template <int TB, int NS>
__device__ __forceinline__ void f32_dx_few(const LmRows& a, const LmPiece& p, const float* __restrict__ w_t, int ld_wt, int slices,
                                           int M, unsigned char* smem) {
  typedef FewRing<float, TB, NS> R;
  const int lane = threadIdx.x & 63, l15 = lane & 15, q = lane >> 4, wave = threadIdx.x >> 6;
  const int i0 = blockIdx.x * R::BV, z = blockIdx.y, all = p.pitch * 4 / ROWB;
  const int k0 = static_cast<int>(static_cast<long long>(all) * z / slices);
  const int nkt = static_cast<int>(static_cast<long long>(all) * (z + 1) / slices) - k0;
  f32x4 acc[2][TB];
  R::run(reinterpret_cast<const unsigned char*>(w_t + static_cast<size_t>(i0) * ld_wt + p.v0) + static_cast<size_t>(k0) * ROWB,
         static_cast<size_t>(ld_wt) * 4, a.d - i0, static_cast<const unsigned char*>(p.e) + static_cast<size_t>(k0) * ROWB,
         [&](int r) { return static_cast<uint32_t>(min(r, M - 1)) * static_cast<uint32_t>(p.pitch * 4); }, nkt, smem, acc);
  float* out = p.acc + static_cast<size_t>(z) * M * a.d + i0 + wave * 32 + 4 * q;   // lane: columns 16 f + r of row 16 b + l15
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int m = 16 * b + l15;
    if (m >= M) continue;
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      f32x4* o = reinterpret_cast<f32x4*>(out + static_cast<size_t>(m) * a.d + 16 * f);
      *o = p.first ? acc[f][b] : a.alpha[p.m0 + m] * *o + acc[f][b];
    }
  }
}

template <int MOST>
__global__ __launch_bounds__(256) void lm_f32_dx_few(LmRows a, LmPiece p, const float* __restrict__ w_t, int ld_wt, int slices) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kFewBytes<MOST>];
  const int M = *p.count;
  if (M == 0) return;
  few_case<MOST>(M, [&](auto tb, auto ns) {
    f32_dx_few<decltype(tb)::value, decltype(ns)::value>(a, p, w_t, ld_wt, slices, M, smem);
  });
}

int lm_tiles(int n) { return (n + 255) / 256; }

template <bool SIX>
hipError_t lm_logits(const LmRows& a, const LmPiece& p, hipStream_t s) {
  const int n = lm_tiles(p.cols) * 256;
  ARows<bf16_t> A{static_cast<const bf16_t*>(a.x), a.idx + p.m0, a.d};
  BRows<bf16_t> B{static_cast<const bf16_t*>(a.w) + static_cast<size_t>(p.v0) * a.d, nullptr, INT_MAX, a.d, p.cols - 1};
  if constexpr (SIX) {
    A = {static_cast<const bf16_t*>(a.xs) + static_cast<size_t>(p.m0) * a.d, nullptr, a.d, nullptr, a.d / BK,
         static_cast<size_t>(a.T) * a.d};
    B.b0 = static_cast<const bf16_t*>(p.ws);
    B.term = static_cast<size_t>(p.cols) * a.d;
  }
  const int K = SIX ? 6 * a.d : a.d;
  if (p.logits) {
    const EpiLmLogits<SIX> epi{{p.logits, p.ldl, static_cast<size_t>(p.rows_max) * p.ldl}, {}};
    return run_phase_split(A, B, epi, p.count, p.rows_max, n, K, p.slices, s);
  }
  const float* ref = a.ref + p.m0;
  const int* tgt = a.tgt + p.m0;
  bf16_t* e = static_cast<bf16_t*>(p.e);
  const size_t term = static_cast<size_t>(p.rows_max) * p.pitch;
  const int parts = p.parts;
  if (e)
    return run_phase<false>(A, B, EpiLmExp<true, SIX>{{}, ref, tgt, p.v0, p.cols, p.pitch, e, term, p.part, parts}, p.count,
                            p.rows_max, n, K, s, false);
  return run_phase<false>(A, B, EpiLmExp<false, SIX>{{}, ref, tgt, p.v0, p.cols, p.pitch, e, term, p.part, parts}, p.count,
                          p.rows_max, n, K, s, false);
}

template <bool SIX>
hipError_t lm_dx(const LmRows& a, const LmPiece& p, const void* w_t, int ld_wt, hipStream_t s) {
  ARows<bf16_t> A{static_cast<const bf16_t*>(p.e), nullptr, p.pitch, nullptr, p.pitch / BK,
                  static_cast<size_t>(p.rows_max) * p.pitch};
  BRows<bf16_t> B{static_cast<const bf16_t*>(w_t) + p.v0, nullptr, INT_MAX, ld_wt};
  if constexpr (SIX) B = {static_cast<const bf16_t*>(p.wts), nullptr, INT_MAX, p.pitch, INT_MAX, nullptr,
                          static_cast<size_t>(a.d) * p.pitch};
  const int n_tiles = a.d / 256, K = SIX ? 6 * p.pitch : p.pitch;
  const int blocks = (std::max((p.rows_max + 127) / 128 * n_tiles, kLmDxBlocks) + 7) / 8 * 8 + 8;
  const float* alpha = a.alpha + p.m0;
  const int* plan = a.plan + p.chunk;
  if (p.first)
    lm_dx_kernel<<<blocks, 512, 0, s>>>(A, B, EpiLmAcc<true, SIX>{{}, p.acc, a.d, alpha}, p.count, plan, p.rows_max, K, n_tiles);
  else
    lm_dx_kernel<<<blocks, 512, 0, s>>>(A, B, EpiLmAcc<false, SIX>{{}, p.acc, a.d, alpha}, p.count, plan, p.rows_max, K, n_tiles);
  return hipGetLastError();
}

template <bool SIX>
hipError_t lm_g(const LmRows& a, int v0, int cols, const void* ws, void* g, int pitch, hipStream_t s) {
  ARows<bf16_t> A{static_cast<const bf16_t*>(a.w) + static_cast<size_t>(v0) * a.d, nullptr, a.d};
  BRows<bf16_t> B{static_cast<const bf16_t*>(a.x), nullptr, INT_MAX, a.d, a.T - 1, a.idx};
  if constexpr (SIX) {
    A = {static_cast<const bf16_t*>(ws), nullptr, a.d, nullptr, a.d / BK, static_cast<size_t>(cols) * a.d};
    B = {static_cast<const bf16_t*>(a.xs), nullptr, INT_MAX, a.d, a.T - 1, nullptr, static_cast<size_t>(a.T) * a.d};
  }
  const EpiLmG<SIX> epi{{}, a.lse, a.own, a.tgt, a.counts, v0, pitch, static_cast<bf16_t*>(g), static_cast<size_t>(cols) * pitch};
  const auto blocks = [&](int bm) { return ((cols + bm - 1) / bm * lm_tiles(pitch) + 7) / 8 * 8; };
  // enough for any choice of any count
  const int grid = std::max({blocks(256), std::min(blocks(192), 8 * kCUs + 8), std::min(blocks(128), 4 * kCUs + 8)});
  lm_g_product<<<grid, 512, 0, s>>>(A, B, epi, cols, SIX ? 6 * a.d : a.d);
  return hipGetLastError();
}

template <typename T, bool SIX>
hipError_t lm_dw(const LmRows& a, int v0, int cols, const void* g, const void* xT, int pitch, void* dw, hipStream_t s) {
  ARows<bf16_t> A{static_cast<const bf16_t*>(g), nullptr, pitch, nullptr, 0, static_cast<size_t>(cols) * pitch};
  BRows<bf16_t> B{static_cast<const bf16_t*>(xT), nullptr, INT_MAX, pitch, INT_MAX, nullptr, static_cast<size_t>(a.d) * pitch};
  const EpiLmDw<T, SIX> epi{{}, static_cast<T*>(dw) + static_cast<size_t>(v0) * a.d, a.d, a.counts, a.scale, a.mean};
  return run_phase<false>(A, B, epi, nullptr, cols, a.d, pitch, s);
}

}  // namespace

// The form that the logits take: the large products with e in their epilogue; where 128-row tiles leave half of the
// CUs idle or more and a workgroup of the combining pass holds a row, K slices of the logits, for that pass to
// exponentiate (134 rows of d = 1536 against 1066 columns: 42 -> 31 us a call).  Few rows against a head of up to
// 160 MB: the streaming form (3 rows of d = 768 against 77287 columns 43 -> 34 us a call, 8 of 2048 against 9000
// 48 -> 37); larger heads draw 5.6 TB/s on the large tiles and 4.8 there (16 rows of 4096 against 128256: 185 and 222 us).
// Longer rows gain nothing from slices: 10 rows of d = 2048 against 39058 columns, 153 tiles, took 56 us so and 65 + 7
// in five slices.  kLmF32: kept, or for few rows the streaming form (28 rows of d = 3840 against 75583 columns 462 ->
// 256 us a call, 4.6 TB/s; 60 of 1024 against 30000 82 -> 54) where its workgroups take most CUs (64 of them: one row of
// 4096 against 8192 45 -> 67).
// fp32 rows that the head, or W^T, streams past: with more than 64 one workgroup fills a CU's LDS, and narrow heads pay
// for its ends (96 rows of d = 1024 against 30000 columns, logits and dx, 327 -> 178 us a call, 127 of 2304 against 45397
// 447 -> 336 the logits; 127 of 512 against 16000 48 and 53).
static bool lm_f32_few(int rows, int d) { return rows <= kLmFewRows || (rows <= kLmFewRowsF32 && d >= 1024); }

LmParts lm_parts(int mode, int rows, int cols, int d) {
  const LmParts few{(cols + 127) / 128, 7, 0};
  if (mode == kLmF32) {
    if (lm_f32_few(rows, d) && (cols + 127) / 128 >= kLmFewF32) return few;
    return cols <= kLmLogitsMax ? LmParts{0, 0, 1} : LmParts{(cols + 8191) / 8192, 13, 1};
  }
  const int tiles = (rows + 127) / 128 * lm_tiles(cols), ktiles = d / 64 * (mode == kLmSplit ? 6 : 1);
  const int S = 2 * tiles > kCUs || cols > kLmLogitsMax - 256 ? 1 : std::min(kCUs / tiles, ktiles / 4);
  if (S > 1) return {0, 0, S};
  if (mode == kLmBf16 && rows <= kLmFewRows && static_cast<long long>(cols) * d <= kLmFewHead) return few;
  return {4 * lm_tiles(cols), 0, 0};
}

hipError_t launch_lm_score_logits(const LmRows& a, const LmPiece& p, hipStream_t s) {
  const int grid = (p.cols + 127) / 128;
#define HERO_LM_SCORE(TYPE)                                                \
  if (a.T <= 16)                                                        \
    lm_logits_few<TYPE, 1, false, true><<<grid, 256, 0, s>>>(a, p);     \
  else if (a.T <= 32)                                                   \
    lm_logits_few<TYPE, 2, false, true><<<grid, 256, 0, s>>>(a, p);     \
  else                                                                  \
    lm_logits_few<TYPE, 4, false, true><<<grid, 256, 0, s>>>(a, p)
  if (a.mode == kLmBf16) {
    HERO_LM_SCORE(bf16_t);
  } else {
    HERO_LM_SCORE(float);
  }
#undef HERO_LM_SCORE
  return hipGetLastError();
}

hipError_t launch_lm_logits(const LmRows& a, const LmPiece& p, hipStream_t s) {
  if (!p.logits && p.shift) {   // the streaming form
    const int grid = (p.cols + 127) / 128;
#define HERO_LM_FEW(T, MOST)                                      \
  (p.e ? lm_logits_few<T, MOST, true><<<grid, 256, 0, s>>>(a, p) \
       : lm_logits_few<T, MOST, false><<<grid, 256, 0, s>>>(a, p))
#define HERO_LM_FEW_ROWS(T)      \
  if (p.rows_max <= 16)          \
    HERO_LM_FEW(T, 1);        \
  else if (p.rows_max <= 32)     \
    HERO_LM_FEW(T, 2);        \
  else if (p.rows_max <= 64)     \
    HERO_LM_FEW(T, 4)
    if (a.mode == kLmBf16) {
      HERO_LM_FEW_ROWS(bf16_t);
    } else {
      HERO_LM_FEW_ROWS(float);
      else if (p.rows_max <= 96)
        HERO_LM_FEW(float, 6);
      else
        HERO_LM_FEW(float, 8);
    }
#undef HERO_LM_FEW_ROWS
#undef HERO_LM_FEW
    return hipGetLastError();
  }
  if (a.mode == kLmBf16) return lm_logits<false>(a, p, s);
  if (a.mode == kLmSplit) return lm_logits<true>(a, p, s);
  return launch_lm_f32_logits(static_cast<const float*>(a.x), a.idx + p.m0, p.count, p.rows_max,
                              static_cast<const float*>(a.w) + static_cast<size_t>(p.v0) * a.d, p.cols, a.d, p.logits, p.ldl, s);
}

// K slices of the streaming dx product, of at least 256 columns each: two workgroups a CU; 0: the other form, whose tiles
// read 64-byte pieces of rows (60 rows of d = 4096 against 128256 columns with the logits 1759 -> 1175 us a call, 60 of 256
// against 100000 176 -> 130; against 10000 of d = 1024 80 and 83)
int lm_f32_few_slices(int rows, int d, int K) {
  if (!lm_f32_few(rows, d) || K < 256 || static_cast<long long>(d) * K < kLmFewDx) return 0;
  return std::max(1, std::min({2 * kCUs / (d / 128), K / 256, 64}));
}

hipError_t launch_lm_dx(const LmRows& a, const LmPiece& p, const void* w_t, int ld_wt, hipStream_t s) {
  if (a.mode == kLmBf16) return lm_dx<false>(a, p, w_t, ld_wt, s);
  if (a.mode == kLmSplit) return lm_dx<true>(a, p, nullptr, 0, s);
  if (a.f32_few) {
    const float* wt = static_cast<const float*>(w_t);
    const dim3 grid(a.d / 128, a.f32_slices);
    if (p.rows_max <= 16)
      lm_f32_dx_few<1><<<grid, 256, 0, s>>>(a, p, wt, ld_wt, a.f32_slices);
    else if (p.rows_max <= 32)
      lm_f32_dx_few<2><<<grid, 256, 0, s>>>(a, p, wt, ld_wt, a.f32_slices);
    else if (p.rows_max <= 64)
      lm_f32_dx_few<4><<<grid, 256, 0, s>>>(a, p, wt, ld_wt, a.f32_slices);
    else if (p.rows_max <= 96)
      lm_f32_dx_few<6><<<grid, 256, 0, s>>>(a, p, wt, ld_wt, a.f32_slices);
    else
      lm_f32_dx_few<8><<<grid, 256, 0, s>>>(a, p, wt, ld_wt, a.f32_slices);
    return hipGetLastError();
  }
  return launch_lm_f32_dx(static_cast<const float*>(p.e), p.count, p.rows_max, p.pitch, static_cast<const float*>(w_t) + p.v0,
                          ld_wt, a.d, a.f32_slices, a.alpha + p.m0, p.first, p.acc, s);
}

// K slices of a dW product whose 128-row tiles leave half of the CUs idle or more: a k-tile takes 0.62 us, the slices
// are written and read at 4.5 TB/s, by one more launch (3300 rows of d = 512 against 1097 columns, 18 tiles: 78 -> 68 us a
// call)
int lm_dw_slices(const LmRows& a, int cols) {
  const int tiles = (cols + 127) / 128 * (a.d / 256);
  if (a.mode == kLmF32 || 2 * tiles > kCUs) return 1;
  const double k = (a.mode == kLmSplit ? 6 : 1) * (a.T / 64) * 0.62, part = 8.0 * cols * a.d / 4.5e6;
  int best = 1;
  double time = k;
  for (int S = 2; S <= kCUs / tiles; ++S)
    if (k / S + part * S + 5.0 < time) {
      time = k / S + part * S + 5.0;
      best = S;
    }
  return lm_dw_slices_of(best, a.T);
}

hipError_t launch_lm_dw_part(const LmRows& a, int cols, const void* g, const void* xT, int pitch, float* part, int slices,
                             hipStream_t s) {
  ARows<bf16_t> A{static_cast<const bf16_t*>(g), nullptr, pitch, nullptr, 0, static_cast<size_t>(cols) * pitch};
  BRows<bf16_t> B{static_cast<const bf16_t*>(xT), nullptr, INT_MAX, pitch, INT_MAX, nullptr, static_cast<size_t>(a.d) * pitch};
  const int n_tiles = a.d / 256;
  const dim3 grid(((cols + 127) / 128 * n_tiles + 7) / 8 * 8, slices);
  if (a.mode == kLmSplit)
    lm_dw_part_kernel<<<grid, 512, 0, s>>>(A, B, EpiLmDwPart<true>{{{}, part, a.d, nullptr}, a.counts}, cols, n_tiles, slices);
  else
    lm_dw_part_kernel<<<grid, 512, 0, s>>>(A, B, EpiLmDwPart<false>{{{}, part, a.d, nullptr}, a.counts}, cols, n_tiles, slices);
  return hipGetLastError();
}

// 98 rows in bf16, four groups of tokens staged: 518 us a call where the large product takes 494.  fp32: all that do not
// take three-term operands.
bool lm_dw_few_rows(int mode, int T) { return mode == kLmBf16 ? T <= 64 : mode == kLmF32 && T <= 128; }

hipError_t launch_lm_dw_few(const LmRows& a, int cols, const void* g, const void* xT, int pitch, void* dw, hipStream_t s) {
  const bool most = a.mode != kLmBf16 && a.T > 64;   // what is staged has to fit
  const int gx = (cols + 127) / 128, width = gx * ((a.d + 255) / 256) >= kCUs ? most ? 128 : 256 : 64;   // small heads: more workgroups
  const dim3 grid(gx, (a.d + width - 1) / width);
#define HERO_LM_DW(T, G)                                                                                       \
  lm_dw_few<T, G><<<grid, 256, 0, s>>>(a, cols, static_cast<const T*>(g), static_cast<const T*>(xT), pitch, width, \
                                       static_cast<T*>(dw))
  if (a.mode == kLmBf16) {
    if (a.T <= 32) HERO_LM_DW(bf16_t, 1);
    else HERO_LM_DW(bf16_t, 2);
  } else {
    if (a.T <= 16) HERO_LM_DW(float, 1);
    else if (a.T <= 32) HERO_LM_DW(float, 2);
    else if (a.T <= 64) HERO_LM_DW(float, 4);
    else HERO_LM_DW(float, 8);
  }
#undef HERO_LM_DW
  return hipGetLastError();
}

hipError_t launch_lm_dw(const LmRows& a, int v0, int cols, const void* g, const void* xT, int pitch, void* dw, hipStream_t s) {
  if (a.mode == kLmBf16) return lm_dw<bf16_t, false>(a, v0, cols, g, xT, pitch, dw, s);
  if (a.mode == kLmSplit) return lm_dw<float, true>(a, v0, cols, g, xT, pitch, dw, s);
  return launch_lm_f32_dw(static_cast<const float*>(g), cols, static_cast<const float*>(xT), a.d, pitch,
                          static_cast<float*>(dw) + static_cast<size_t>(v0) * a.d, s);
}

hipError_t launch_lm_g_products(const LmRows& a, int v0, int cols, const void* ws, void* g, int pitch, hipStream_t s) {
  return a.mode == kLmSplit ? lm_g<true>(a, v0, cols, ws, g, pitch, s) : lm_g<false>(a, v0, cols, ws, g, pitch, s);
}

}  // namespace hero
