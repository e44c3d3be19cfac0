// Language-model loss over a vocabulary, in pieces, with its gradients; the logits are not kept.
//
//   l_tv = <x_t, W_v>, y the token's target, S_t = sum over v != y of exp(l_tv - l_ty)
//   nll_t = log(1 + S_t)
//   dx_t  = c / (1 + S_t) (sum over v != y of exp(l_tv - l_ty) W_v - S_t W_y)
//   dW_v  = c sum over t of (p_tv - [v = y_t]) x_t,   c = scale, or scale / N for the mean of N tokens
//
// Written over the other columns, neither the loss nor the gradient of a token that the model is sure of
// is a difference of close numbers.  The target's logit, found by a dot product before anything else,
// is the reference of all exponentials, which is why one pass over the vocabulary is enough: a row's sums
// and its sum of e W are gathered piece by piece and divided at the end.  A row whose logits rise more
// than e^60 above its target changes its reference on the way (EpiLmExp, the combining pass).
//
// Tokens without a target cost nothing: the rows that count are compacted on the device, and every product
// takes their number from there.  The passes here are short and read what the products left in the caches;
// the products (k_lm_gemm.hip) bound the whole, launches and latencies the smallest calls.
#include <limits.h>

#include <algorithm>

#include "hero_device.h"
#include "hero_kernels.h"

namespace hero {
namespace {

constexpr int kRowsThreads = 1024;

// Tile height and K slices of the dx products of M rows, by one wave, a candidate a lane and turn: the time in
// rounds of workgroups over the CUs, a round weighted by its height (as phase_rows) and by its k-tiles, of which
// storing an fp32 tile takes about twelve, and the finishing pass's reading of all slices at 4 TB/s, at least 0.15 us
// each (125 is a k-tile of 256 rows, 1.45 us).  2048 rows of d = 4096 against 32768 columns: 128-row tiles in one
// round 443 us, 256-row tiles in two slices 399.
__device__ __forceinline__ int dx_plan(const LmRows& a, int M, int lane) {
  float time = 3.0e38f;
  int best = 256 | 1 << 16;
  for (int c = lane; c < 3 * 19; c += kWave) {   // 1, 2, 4 or 8, 16 .. 128 slices: whole XCDs to a slice
    const int bm = 256 - 64 * (c % 3), k = c / 3, S = k < 4 ? 1 << k : 8 * (k - 2), w = bm == 256 ? 125 : bm == 192 ? 100 : 75;
    const int tiles = (M + bm - 1) / bm * a.dx_tiles;
    if (S > 1 && (static_cast<long long>(S) * M > a.acc_rows || tiles * S > kLmDxBlocks || a.dx_depth < 4 * S)) continue;
    const float v = static_cast<float>((tiles * S + 255) / 256 * w) * (static_cast<float>(a.dx_depth) / S + 12.f) +
                    static_cast<float>(S) * (static_cast<float>(M) * a.d * (125.f * 4.f / (1.45f * 4.0e6f)) + 13.f);
    if (v < time) {
      time = v;
      best = bm | S << 16;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const float v = __shfl_xor(time, off, kWave);
    const int b = __shfl_xor(best, off, kWave);
    if (v < time || (v == time && b < best)) {
      time = v;
      best = b;
    }
  }
  return best;
}

__device__ __forceinline__ void write_plan(const LmRows& a, int c, int rows, int lane) {
  const int plan = a.mode == kLmF32 ? 128 | a.f32_slices << 16 : a.acc_rows == 0 ? 0 : dx_plan(a, rows, lane);
  if (lane == 0) {
    a.counts[1 + c] = rows;
    a.plan[c] = plan;
  }
}

// The target's logit of row m, token t, by one wave
template <typename T>
__device__ __forceinline__ void target_row(const LmRows& a, int m, int t, int lane) {
  const int y = a.targets[t];
  const T* x = static_cast<const T*>(a.x) + static_cast<size_t>(t) * a.d;
  const T* w = static_cast<const T*>(a.w) + static_cast<size_t>(y) * a.d;
  float s = 0.f;
#pragma unroll 4
  for (int c = lane; c < a.d / 8; c += kWave) {
    Raw8<T> p, q;
    p.load(x + 8 * c);
    q.load(w + 8 * c);
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fmaf(p[k], q[k], s);
  }
  s = wave_sum(s);
  if (lane == 0) {
    a.tgt[m] = y;
    a.lt[m] = s;
    a.ref[m] = s - s == 0.f ? s : __uint_as_float(0x7fc00000u);   // an infinite logit leaves no finite loss
    a.sum[m] = 0.f;
  }
}

// four targets from t on; those behind the last token do not count
__device__ __forceinline__ int4 four_targets(const LmRows& a, int t) {
  if (t + 4 <= a.T) return *reinterpret_cast<const int4*>(a.targets + t);
  return int4{t < a.T ? a.targets[t] : -1, t + 1 < a.T ? a.targets[t + 1] : -1, t + 2 < a.T ? a.targets[t + 2] : -1, -1};
}
__device__ __forceinline__ int counted(const LmRows& a, int y) {
  return static_cast<unsigned>(y) < static_cast<unsigned>(a.vocab);
}

// Up to kLmSmall tokens in one launch: every workgroup counts all targets for itself, F fours a thread, and takes
// one of them, a token a wave.  5719 tokens of d = 512: 6 us, where a compaction by one workgroup and a second launch
// took 14 + 4.
template <typename T, int F>
__global__ __launch_bounds__(256) void lm_rows_small_kernel(LmRows a) {
  __shared__ int wsum[4], rank[4], live[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t0 = 4 * F * threadIdx.x;
  int in[F], n = 0;   // four bits a four
#pragma unroll
  for (int f = 0; f < F; ++f) {
    const int4 y = four_targets(a, t0 + 4 * f);
    in[f] = counted(a, y.x) | counted(a, y.y) << 1 | counted(a, y.z) << 2 | counted(a, y.w) << 3;
    n += __popc(in[f]);
  }
  int incl = n;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int v = __shfl_up(incl, off, kWave);
    if (lane >= off) incl += v;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  const int total = wsum[0] + wsum[1] + wsum[2] + wsum[3];
  if (threadIdx.x == blockIdx.x / F) {
    int m = incl - n;
    for (int w = 0; w < wave; ++w) m += wsum[w];
    int bits = 0;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      if (f < static_cast<int>(blockIdx.x % F)) m += __popc(in[f]);
      if (f == static_cast<int>(blockIdx.x % F)) bits = in[f];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      live[k] = bits >> k & 1;
      rank[k] = m;
      m += live[k];
    }
  }
  if (blockIdx.x == 0) {
    if (wave == 3) {
      if (lane == 0) {
        a.counts[0] = total;
        *a.done = 0;
      }
      write_plan(a, 0, total, lane);
    }
    for (int i = total + threadIdx.x; i < a.T; i += 256) a.idx[i] = 0;   // rows that no result uses
  }
  __syncthreads();
  const int t = 4 * blockIdx.x + wave, m = rank[wave];
  if (t >= a.T) return;
  if (!live[wave]) {
    if (lane == 0) {
      a.inv[t] = -1;
      if (a.token_loss) a.token_loss[t] = 0.f;
    }
    return;
  }
  if (lane == 0) {
    a.inv[t] = m;
    a.idx[m] = t;
  }
  target_row<T>(a, m, t, lane);
}

// More tokens: ordered compaction by one workgroup, a run of neighbouring tokens per thread, then a wave a row.
__global__ __launch_bounds__(kRowsThreads) void lm_rows_kernel(LmRows a) {
  __shared__ int wsum[kRowsThreads / kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (a.T + 4 * kRowsThreads - 1) / (4 * kRowsThreads) * 4;   // whole 16-byte loads
  const int t0 = min(a.T, static_cast<int>(threadIdx.x) * per), t1 = min(a.T, t0 + per);
  int n = 0;
#pragma unroll 4
  for (int t = t0; t < t1; t += 4) {
    const int4 y = four_targets(a, t);
    n += counted(a, y.x) + counted(a, y.y) + counted(a, y.z) + counted(a, y.w);
  }
  int incl = n;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int v = __shfl_up(incl, off, kWave);
    if (lane >= off) incl += v;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int m = incl - n, total = 0;
  for (int w = 0; w < kRowsThreads / kWave; ++w) {
    if (w < wave) m += wsum[w];
    total += wsum[w];
  }
#pragma unroll 2
  for (int t = t0; t < t1; t += 4) {
    const int4 y = four_targets(a, t);
    const int v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (t + k >= t1) break;
      const bool in = counted(a, v[k]);
      a.inv[t + k] = in ? m : -1;
      if (in)
        a.idx[m++] = t + k;
      else if (a.token_loss)
        a.token_loss[t + k] = 0.f;
    }
  }
  for (int i = total + threadIdx.x; i < a.T; i += kRowsThreads) a.idx[i] = 0;   // rows that no result uses
  if (threadIdx.x == 0) a.counts[0] = total;
  for (int c = wave; c < a.n_chunks; c += kRowsThreads / kWave)
    write_plan(a, c, max(0, min(a.chunk, total - c * a.chunk)), lane);
}

template <typename T>
__global__ __launch_bounds__(256) void lm_targets_kernel(LmRows a) {
  const int m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m < a.counts[0]) target_row<T>(a, m, a.idx[m], threadIdx.x & 63);
}

// eight values of a row: bf16, fp32, or so many bf16 terms
template <int MODE, int TERMS = MODE == kLmSplit ? 3 : 1>
__device__ __forceinline__ void put8(void* base, size_t at, size_t term, const float* v) {
  if constexpr (MODE == kLmF32) {
    st8(static_cast<float*>(base) + at, v);
  } else {
    float r[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) r[k] = v[k];
    for (int t = 0; t < TERMS; ++t) {
      st8(static_cast<bf16_t*>(base) + at + t * term, r);
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] -= bf16_to_f32(f32_to_bf16(r[k]));
    }
  }
}

// sum and maximum over a workgroup of NT threads, in every thread
template <int NT>
__device__ __forceinline__ float group_reduce(float v, bool maximum, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const float o = __shfl_xor(v, off, kWave);
    v = maximum ? fmaxf(v, o) : v + o;
  }
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / kWave; ++w) v = maximum ? fmaxf(v, red[w]) : v + red[w];
  __syncthreads();
  return v;
}

// The sums of a row after a piece, by thread 0 of its workgroup; after the last piece its loss.
__device__ __forceinline__ void row_sums(const LmRows& a, const LmPiece& p, int m, float r0, float r, float s) {
  const float f0 = r > r0 ? expf(r0 - r) : 1.0f;
  s = fmaf(a.sum[m], f0, s);
  a.sum[m] = s;
  a.alpha[m] = f0;
  a.ref[m] = r;
  if (!p.last) return;
  // s is in units of e^ref
  const float lt = a.lt[m], own = lt == r ? 1.0f : expf(lt - r);
  const float nll = lt == r ? log1pf(s) : logf(s + own) + (r - lt);
  // read by another workgroup of this launch (add_losses): past the XCD's own cache
  __hip_atomic_store(a.nll + m, nll, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (a.token_loss) a.token_loss[a.idx[m]] = nll;
  a.lse[m] = lt + nll;
  a.own[m] = -s / (s + own);
}

__device__ __forceinline__ void add_losses(const LmRows& a) {
  __shared__ double red[16];
  const int N = a.counts[0];
  double s = 0.0;
  for (int m = threadIdx.x; m < N; m += blockDim.x)
    s += static_cast<double>(__hip_atomic_load(a.nll + m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < static_cast<int>(blockDim.x) / kWave; ++w) s += red[w];
    a.loss[0] = static_cast<float>(a.scale * (a.mean ? s / max(N, 1) : s));
  }
}

// Few tokens: the workgroup whose row is the last to finish adds the losses, in row order, which saves a launch
// (5 us of 36 where one token is scored).  Without rows the first workgroup writes the loss of none.  Only the
// rows' losses pass between workgroups, by device-scope stores that are waited for before the count: a
// device-scope fence instead writes every dirty line of the XCD's cache back (1000 rows 55 us, so 20).  More rows
// than kLmCounted queue at the counter for longer than a launch takes.
__device__ __forceinline__ void row_done(const LmRows& a, const LmPiece& p) {
  __shared__ bool last;
  if (a.T > kLmCounted || !p.last) return;
  if (threadIdx.x == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 ==
           static_cast<unsigned>(a.counts[0]);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __syncthreads();
  if (last) add_losses(a);
}
__device__ __forceinline__ bool no_row(const LmRows& a, const LmPiece& p, int i) {
  if (i < *p.count) return false;
  if (i == 0 && p.last && a.T <= kLmCounted && threadIdx.x == 0) a.loss[0] = 0.f;
  return true;
}

__global__ __launch_bounds__(1024) void lm_sum_kernel(LmRows a) { add_losses(a); }

// The sums of a row's parts, a workgroup a row.  A part whose reference is not the row's (a logit far above the
// target's) raises the row's: then the earlier sums, and this piece's e, are rescaled.
__global__ __launch_bounds__(256) void lm_combine_kernel(LmRows a, LmPiece p) {
  __shared__ float red[4];
  const int parts = p.parts, i = blockIdx.x, m = p.m0 + i;
  if (no_row(a, p, i)) return;
  const float r0 = a.ref[m];
  const float2* part = p.part + static_cast<size_t>(i) * parts;
  float r = r0;
  float s = 0.f;
  for (int q = threadIdx.x; q < parts; q += 256) {
    const float2 v = part[q];
    r = fmaxf(r, v.x);
    s += v.y;
  }
  r = group_reduce<256>(r, true, red);
  const bool raised = r > r0;
  if (raised) {
    s = 0.f;
    for (int q = threadIdx.x; q < parts; q += 256) s += part[q].y * expf(part[q].x - r);
  }
  s = group_reduce<256>(s, false, red);
  if (threadIdx.x == 0) row_sums(a, p, m, r0, r, s);
  if (raised && p.e) {
    bf16_t* e = static_cast<bf16_t*>(p.e) + static_cast<size_t>(i) * p.pitch;
    float* e32 = static_cast<float*>(p.e) + static_cast<size_t>(i) * p.pitch;
    const size_t term = a.mode == kLmSplit ? static_cast<size_t>(p.rows_max) * p.pitch : 0;
    for (int n = threadIdx.x; n < p.pitch; n += 256) {
      const int q = p.shift ? n >> p.shift : (n >> 8) * 4 + ((n & 127) >> 5);
      // in two halves: e may be e^60 and the factor below the smallest number
      const float f = expf(0.5f * (part[q].x - r));
      if (a.mode == kLmF32) {
        e32[n] = e32[n] * f * f;
      } else if (term == 0) {
        e[n] = f32_to_bf16(bf16_to_f32(e[n]) * f * f);
      } else {
        float v = (bf16_to_f32(e[n]) + bf16_to_f32(e[n + term]) + bf16_to_f32(e[n + 2 * term])) * f * f;
        for (int t = 0; t < 3; ++t) {
          e[n + t * term] = f32_to_bf16(v);
          v -= bf16_to_f32(e[n + t * term]);
        }
      }
    }
  }
  row_done(a, p);
}

// The losses of few tokens, a workgroup a token: the target's logit, then the sums of the parts, each in units of its own
// maximum, taken to that logit (or to the row's maximum, 60 above it).  The last workgroup adds the losses.  Three tokens
// against 77287 columns of d = 768 29.9 us a call, with the rows' launch and the combining pass 34.1.
template <typename T>
__global__ __launch_bounds__(256) void lm_score_kernel(LmRows a, LmPiece p) {
  __shared__ float red[4];
  __shared__ bool last;
  const int t = blockIdx.x, y = a.targets[t];
  float nll = 0.f;
  if (static_cast<unsigned>(y) < static_cast<unsigned>(a.vocab)) {
    const T* x = static_cast<const T*>(a.x) + static_cast<size_t>(t) * a.d;
    const T* w = static_cast<const T*>(a.w) + static_cast<size_t>(y) * a.d;
    const float2* part = p.part + static_cast<size_t>(t) * p.parts;
    float lt = 0.f, top = -INFINITY;
    for (int c = threadIdx.x; c < a.d / 8; c += 256) {
      Raw8<T> u, v;
      u.load(x + 8 * c);
      v.load(w + 8 * c);
#pragma unroll
      for (int k = 0; k < 8; ++k) lt = fmaf(u[k], v[k], lt);
    }
    for (int q = threadIdx.x; q < p.parts; q += 256)
      if (!(part[q].y == 0.f)) top = fmaxf(top, part[q].x);   // nothing but the target, or -infinities: no reference
    lt = group_reduce<256>(lt, false, red);
    top = group_reduce<256>(top, true, red);
    if (!(lt - lt == 0.f)) lt = __uint_as_float(0x7fc00000u);   // an infinite logit leaves no finite loss
    const float r = top - lt > 60.0f ? top : lt;
    float s = 0.f;
    for (int q = threadIdx.x; q < p.parts; q += 256) s = fmaf(part[q].y, expf(part[q].x - r), s);
    s = group_reduce<256>(s, false, red);
    nll = lt == r ? log1pf(s) : logf(s + expf(lt - r)) + (r - lt);
  }
  if (threadIdx.x == 0) {
    if (a.token_loss) a.token_loss[t] = nll;
    __hip_atomic_store(a.nll + t, nll, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    last = __hip_atomic_fetch_add(a.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == static_cast<unsigned>(a.T);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __syncthreads();
  if (!last || threadIdx.x >= 64) return;
  // one wave, at most a token a lane; of a token that does not count a zero
  double sum = 0.0;
  int n = 0;
  if (static_cast<int>(threadIdx.x) < a.T) {
    sum = static_cast<double>(__hip_atomic_load(a.nll + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    n = counted(a, a.targets[threadIdx.x]);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    sum += __shfl_xor(sum, off, kWave);
    n += __shfl_xor(n, off, kWave);
  }
  if (threadIdx.x == 0) a.loss[0] = static_cast<float>(a.scale * (a.mean ? sum / max(n, 1) : sum));
}

// The logits of a piece, in K slices, to e: a workgroup a row, eight columns a thread in registers; zeros up to
// the pitch.  One round of loads, two reductions: reading the logits once for the maximum and once for the
// exponentials took 1088 rows of 1286 columns 11.6 us.  Long fp32 rows: a workgroup 8192 columns (grid y), which are
// a part each for the combining pass (one row of 82971 by one workgroup: 30 us).
template <int MODE, int NT>
__global__ __launch_bounds__(NT) void lm_exp_kernel(LmRows a, LmPiece p) {
  __shared__ float red[16];
  const int i = blockIdx.x, m = p.m0 + i, n = 8 * (blockIdx.y * NT + threadIdx.x);
  if (p.shift ? i >= *p.count : no_row(a, p, i)) return;
  const float* l = p.logits + static_cast<size_t>(i) * p.ldl + n;
  const size_t slice = static_cast<size_t>(p.rows_max) * p.ldl;
  const float r0 = a.ref[m];
  const int tgt = a.tgt[m] - p.v0 - n;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  float top = r0;
  if (n < p.cols) {
    ld8(l, v);
#pragma unroll 4
    for (int z = 1; z < p.slices; ++z) {
      float w[8];
      ld8(l + z * slice, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += w[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (n + k < p.cols) top = fmaxf(top, v[k]);
  }
  top = group_reduce<NT>(top, true, red);
  // the target's logit is a good reference unless the row rises far above it
  const float r = top - r0 > 60.0f ? top : r0;
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = n + k < p.cols && k != tgt ? expf(v[k] - r) : 0.f;
    s += v[k];
  }
  if (p.e && n < p.pitch)
    put8<MODE>(p.e, static_cast<size_t>(i) * p.pitch + n, static_cast<size_t>(p.rows_max) * p.pitch, v);
  s = group_reduce<NT>(s, false, red);
  if (p.shift) {
    if (threadIdx.x == 0) p.part[static_cast<size_t>(i) * p.parts + blockIdx.y] = {r, s};
    return;
  }
  if (threadIdx.x == 0) row_sums(a, p, m, r0, r, s);
  row_done(a, p);
}

// dx: 2048 columns a workgroup, eight a thread, the K slices added in order.  A call of one chunk takes a token a
// workgroup; of several, a row of the chunk, and with the last chunk the tokens without a row behind those.
template <typename T>
__global__ __launch_bounds__(256) void lm_finish_kernel(LmRows a, LmPiece p, T* __restrict__ dx) {
  const int b = blockIdx.x, c = 8 * (blockIdx.y * blockDim.x + threadIdx.x);
  if (c >= a.d) return;
  int t = b, m = 0;
  if (a.n_chunks == 1) {
    m = a.inv[t];
  } else if (b < p.rows_max) {
    if (b >= *p.count) return;
    m = p.m0 + b;
    t = a.idx[m];
  } else {
    t = b - p.rows_max;
    if (a.inv[t] >= 0) return;
    m = -1;
  }
  T* out = dx + static_cast<size_t>(t) * a.d + c;
  if (m < 0) {
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    st8(out, zero);
    return;
  }
  const int S = a.plan[p.chunk] >> 16;
  const size_t stride = static_cast<size_t>(*p.count) * a.d;
  const float* acc = p.acc + static_cast<size_t>(m - p.m0) * a.d + c;
  Raw8<T> w;
  w.load(static_cast<const T*>(a.w) + static_cast<size_t>(a.tgt[m]) * a.d + c);
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int z = 0; z < S; ++z) {
    Raw8<float> v;
    v.load(acc + z * stride);
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] += v[k];
  }
  const float lt = a.lt[m], ref = a.ref[m], s = a.sum[m], inv = 1.0f / (s + (lt == ref ? 1.0f : expf(lt - ref)));
  const float unit = a.mean ? a.scale / static_cast<float>(a.counts[0]) : a.scale;
#pragma unroll
  for (int k = 0; k < 8; ++k) o[k] = unit * ((o[k] - s * w[k]) * inv);
  st8(out, o);
}

// ---------------------------------------------------------------------------
// transposes through 64 x 64 tiles, eight elements a thread on both sides
// ---------------------------------------------------------------------------

__device__ __forceinline__ int depth_of(int rows) { return max(128, (rows + 63) / 64 * 64); }

// dW from its K slices (as many as the counted tokens have work for), eight elements a thread
template <typename T>
__global__ __launch_bounds__(256) void lm_dw_sum_kernel(LmRows a, const float* __restrict__ part, int slices, size_t n,
                                                        T* __restrict__ dw) {
  const size_t e = (static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (e >= n) return;
  const int S = lm_dw_slices_of(slices, depth_of(a.counts[0]));
  const float unit = a.mean ? a.scale / static_cast<float>(max(a.counts[0], 1)) : a.scale;
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int z = 0; z < S; ++z) {
    float v[8];
    ld8(part + z * n + e, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] += v[k];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) o[k] *= unit;
  st8(dw + e, o);
}

// in(r, c, v): the eight values of row r at columns c .. c + 7; out(c, r, v): those of column c at rows r ..
// The kernel owns the tile: with one in each of the two transposes that share a launch half as many workgroups fit a
// CU (1777 tokens of 50257 columns: 63 us, with the one about 47).
typedef float Tile64[64][65];
template <class In, class Out>
__device__ __forceinline__ void transpose64(Tile64& tile, In in, Out out) {
#pragma unroll
  for (int q = threadIdx.x; q < 512; q += 256) {
    float v[8];
    in(q >> 3, 8 * (q & 7), v);
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[q >> 3][8 * (q & 7) + k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int q = threadIdx.x; q < 512; q += 256) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = tile[8 * (q & 7) + k][q >> 3];
    out(q >> 3, 8 * (q & 7), v);
  }
}

// One 64 x 64 tile of xT[i][m] = x[idx[m]][i], zero behind the counted rows as far as the dW product reads
template <int MODE>
__device__ __forceinline__ void xT_tile(Tile64& tile, const LmRows& a, void* __restrict__ xT, int pitch, int i0,
                                        int m0) {
  typedef std::conditional_t<MODE == kLmBf16, bf16_t, float> T;
  const int N = a.counts[0];
  if (MODE != kLmF32 && m0 >= depth_of(N)) return;
  transpose64(
      tile,
      [&](int r, int c, float* v) {
        if (m0 + r < N) {
          ld8(static_cast<const T*>(a.x) + static_cast<size_t>(a.idx[m0 + r]) * a.d + i0 + c, v);
        } else {
          for (int k = 0; k < 8; ++k) v[k] = 0.f;
        }
      },
      [&](int c, int r, const float* v) {
        put8<MODE>(xT, static_cast<size_t>(i0 + c) * pitch + m0 + r, static_cast<size_t>(a.d) * pitch, v);
      });
}

// One 64 x 64 tile of g[n][m] = p - [n = target]: from e of the whole vocabulary (OF_E), or from fp32 logits;
// kLmF32: times the unit.  A bf16 e is divided by its row's sum and rounded a second time, which saves forming the
// logits again (1777 tokens of d = 1024, vocabulary 50257: 196 us); the target's entry is exact but for its own rounding.
// TWO (few rows): two bf16 terms.  With few tokens the rounding of a target's p - 1 is one factor on all of a row of
// dW and does not average out: dW of one token was off by up to 2.4 times its output's rounding, so by 1.4.
template <int MODE, bool OF_E, bool TWO = false>
__device__ __forceinline__ void g_tile(Tile64& tile, const LmRows& a, int v0, int cols, const void* __restrict__ src,
                                       int ld, size_t src_term, void* __restrict__ g, int pitch, int n0, int m0) {
  __shared__ float row[2][64];
  __shared__ int tgt[64];
  const int N = a.counts[0];
  if (MODE != kLmF32 && m0 >= depth_of(N)) return;
  const float unit = MODE != kLmF32 ? 1.0f : a.mean ? a.scale / static_cast<float>(max(N, 1)) : a.scale;
  if (threadIdx.x < 64) {
    const int m = m0 + threadIdx.x;
    const bool in = m < N;
    const float lt = in ? a.lt[m] : 0.f, ref = in ? a.ref[m] : 0.f;
    row[0][threadIdx.x] = !in ? 0.f : OF_E ? unit / (a.sum[m] + (lt == ref ? 1.0f : expf(lt - ref))) : a.lse[m];
    row[1][threadIdx.x] = in ? unit * a.own[m] : 0.f;
    tgt[threadIdx.x] = in ? a.tgt[m] - v0 : INT_MIN;
  }
  __syncthreads();
  transpose64(
      tile,
      [&](int r, int c, float* v) {
        if (m0 + r >= N || n0 + c >= ld) {
          for (int k = 0; k < 8; ++k) v[k] = 0.f;
          return;
        }
        const size_t at = static_cast<size_t>(m0 + r) * ld + n0 + c;
        const float f = row[0][r];
        if constexpr (MODE == kLmF32) {
          ld8(static_cast<const float*>(src) + at, v);
        } else {
          ld8(static_cast<const bf16_t*>(src) + at, v);
          if constexpr (MODE == kLmSplit)
            for (int t = 1; t < 3; ++t) {
              float w[8];
              ld8(static_cast<const bf16_t*>(src) + at + t * src_term, w);
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] += w[k];
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          v[k] = OF_E ? v[k] * f : unit * expf(v[k] - f);
          if (n0 + c + k == tgt[r]) v[k] = row[1][r];
        }
      },
      [&](int c, int r, const float* v) {
        if (n0 + c < cols)
          put8<MODE, TWO ? 2 : MODE == kLmSplit ? 3 : 1>(g, static_cast<size_t>(n0 + c) * pitch + m0 + r,
                                                         static_cast<size_t>(cols) * pitch, v);
      });
}

template <int MODE>
__global__ __launch_bounds__(256) void lm_xT_kernel(LmRows a, void* __restrict__ xT, int pitch) {
  __shared__ Tile64 tile;
  xT_tile<MODE>(tile, a, xT, pitch, blockIdx.x * 64, blockIdx.y * 64);
}

template <int MODE>
__global__ __launch_bounds__(256) void lm_g_kernel(LmRows a, int v0, int cols, const float* __restrict__ logits, int ld,
                                                   void* __restrict__ g, int pitch) {
  __shared__ Tile64 tile;
  g_tile<MODE, false>(tile, a, v0, cols, logits, ld, 0, g, pitch, blockIdx.x * 64, blockIdx.y * 64);
}

// both operands of the dW product of a call of one piece and one chunk: the first workgroups of a row xT, the rest g
template <int MODE, bool TWO>
__global__ __launch_bounds__(256) void lm_g_of_e_kernel(LmRows a, LmPiece p, void* __restrict__ g, void* __restrict__ xT,
                                                        int pitch) {
  __shared__ Tile64 tile;
  const int nx = a.d / 64, b = blockIdx.x;
  if (b < nx)
    xT_tile<MODE>(tile, a, xT, pitch, b * 64, blockIdx.y * 64);
  else
    g_tile<MODE, true, TWO>(tile, a, 0, p.cols, p.e, p.pitch, static_cast<size_t>(p.rows_max) * p.pitch, g, pitch,
                            (b - nx) * 64, blockIdx.y * 64);
}

// w_t[i][v] = w[v][i], zero from the vocabulary to the pitch (a multiple of 64)
template <typename T>
__global__ __launch_bounds__(256) void lm_head_kernel(const T* __restrict__ w, int vocab, int d, T* __restrict__ w_t,
                                                      int pitch) {
  __shared__ Tile64 tile;
  const int i0 = blockIdx.x * 64, v0 = blockIdx.y * 64;
  transpose64(
      tile,
      [&](int r, int c, float* v) {
        if (v0 + r < vocab) {
          ld8(w + static_cast<size_t>(v0 + r) * d + i0 + c, v);
        } else {
          for (int k = 0; k < 8; ++k) v[k] = 0.f;
        }
      },
      [&](int c, int r, const float* v) { st8(w_t + static_cast<size_t>(i0 + c) * pitch + v0 + r, v); });
}

__global__ __launch_bounds__(256) void lm_terms_kernel(const float* __restrict__ in, int ld_in, const int* __restrict__ idx,
                                                       const int* __restrict__ count, int cols, size_t term,
                                                       bf16_t* __restrict__ out) {
  const int r = blockIdx.x, c = 8 * (blockIdx.y * 256 + threadIdx.x);
  if ((count && r >= *count) || c >= cols) return;
  float v[8];
  ld8(in + static_cast<size_t>(idx ? idx[r] : r) * ld_in + c, v);
  put8<kLmSplit>(out, static_cast<size_t>(r) * cols + c, term, v);
}

// a row of few columns takes few threads, so that more rows are under way
template <int MODE>
void lm_exp(const LmRows& a, const LmPiece& p, hipStream_t s) {
  if (p.pitch <= 2048)
    lm_exp_kernel<MODE, 256><<<p.rows_max, 256, 0, s>>>(a, p);
  else
    lm_exp_kernel<MODE, 1024><<<dim3(p.rows_max, (p.pitch + 8191) / 8192), 1024, 0, s>>>(a, p);
}

}  // namespace

hipError_t launch_lm_rows(const LmRows& a, hipStream_t s) {
  const bool b16 = a.mode == kLmBf16;
  if (a.T <= kLmSmall) {
    const int grid = (a.T + 3) / 4;
#define HERO_LM_ROWS(F)                                                    \
  (b16 ? lm_rows_small_kernel<bf16_t, F><<<grid, 256, 0, s>>>(a) \
       : lm_rows_small_kernel<float, F><<<grid, 256, 0, s>>>(a))
    if (a.T <= 1024)
      HERO_LM_ROWS(1);
    else if (a.T <= 2048)
      HERO_LM_ROWS(2);
    else if (a.T <= 4096)
      HERO_LM_ROWS(4);
    else
      HERO_LM_ROWS(8);
#undef HERO_LM_ROWS
    return hipGetLastError();
  }
  lm_rows_kernel<<<1, kRowsThreads, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (b16)
    lm_targets_kernel<bf16_t><<<(a.T + 3) / 4, 256, 0, s>>>(a);
  else
    lm_targets_kernel<float><<<(a.T + 3) / 4, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_sum(const LmRows& a, hipStream_t s) {
  lm_sum_kernel<<<1, 1024, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_combine(const LmRows& a, const LmPiece& p, hipStream_t s) {
  if (p.logits) {
    if (a.mode == kLmBf16)
      lm_exp<kLmBf16>(a, p, s);
    else if (a.mode == kLmF32)
      lm_exp<kLmF32>(a, p, s);
    else
      lm_exp<kLmSplit>(a, p, s);
  }
  if (!p.logits || p.shift) lm_combine_kernel<<<p.rows_max, 256, 0, s>>>(a, p);
  return hipGetLastError();
}

hipError_t launch_lm_score(const LmRows& a, const LmPiece& p, hipStream_t s) {
  static_assert(kLmFewRows <= kWave, "the losses are added by one wave");
  if (a.mode == kLmBf16)
    lm_score_kernel<bf16_t><<<a.T, 256, 0, s>>>(a, p);
  else
    lm_score_kernel<float><<<a.T, 256, 0, s>>>(a, p);
  return hipGetLastError();
}

hipError_t launch_lm_finish(const LmRows& a, const LmPiece& p, void* dx, hipStream_t s) {
  const int nt = std::min(256, (a.d / 8 + 63) / 64 * 64);
  const int rows = a.n_chunks == 1 ? a.T : p.chunk == a.n_chunks - 1 ? p.rows_max + a.T : p.rows_max;
  const dim3 grid(rows, (a.d / 8 + nt - 1) / nt);
  if (a.mode == kLmBf16)
    lm_finish_kernel<bf16_t><<<grid, nt, 0, s>>>(a, p, static_cast<bf16_t*>(dx));
  else
    lm_finish_kernel<float><<<grid, nt, 0, s>>>(a, p, static_cast<float*>(dx));
  return hipGetLastError();
}

hipError_t launch_lm_xT(const LmRows& a, void* xT, int pitch, hipStream_t s) {
  const dim3 grid(a.d / 64, pitch / 64);
  if (a.mode == kLmBf16)
    lm_xT_kernel<kLmBf16><<<grid, 256, 0, s>>>(a, xT, pitch);
  else if (a.mode == kLmF32)
    lm_xT_kernel<kLmF32><<<grid, 256, 0, s>>>(a, xT, pitch);
  else
    lm_xT_kernel<kLmSplit><<<grid, 256, 0, s>>>(a, xT, pitch);
  return hipGetLastError();
}

hipError_t launch_lm_g(const LmRows& a, int v0, int cols, const void* ws, const float* logits, int ldl, void* g, int pitch,
                       hipStream_t s) {
  if (a.mode != kLmF32) return launch_lm_g_products(a, v0, cols, ws, g, pitch, s);
  lm_g_kernel<kLmF32><<<dim3((cols + 63) / 64, pitch / 64), 256, 0, s>>>(a, v0, cols, logits, ldl, g, pitch);
  return hipGetLastError();
}

hipError_t launch_lm_g_of_e(const LmRows& a, const LmPiece& p, void* g, void* xT, int pitch, hipStream_t s) {
  const dim3 grid(a.d / 64 + (p.cols + 63) / 64, pitch / 64);
  if (a.mode == kLmBf16 && lm_dw_few_rows(a.mode, a.T))
    lm_g_of_e_kernel<kLmBf16, true><<<grid, 256, 0, s>>>(a, p, g, xT, pitch);
  else if (a.mode == kLmBf16)
    lm_g_of_e_kernel<kLmBf16, false><<<grid, 256, 0, s>>>(a, p, g, xT, pitch);
  else if (a.mode == kLmF32)
    lm_g_of_e_kernel<kLmF32, false><<<grid, 256, 0, s>>>(a, p, g, xT, pitch);
  else
    lm_g_of_e_kernel<kLmSplit, false><<<grid, 256, 0, s>>>(a, p, g, xT, pitch);
  return hipGetLastError();
}

hipError_t launch_lm_dw_sum(const LmRows& a, const float* part, int slices, int cols, void* dw, hipStream_t s) {
  const size_t n = static_cast<size_t>(cols) * a.d;
  const int blocks = static_cast<int>((n / 8 + 255) / 256);
  if (a.mode == kLmBf16)
    lm_dw_sum_kernel<bf16_t><<<blocks, 256, 0, s>>>(a, part, slices, n, static_cast<bf16_t*>(dw));
  else
    lm_dw_sum_kernel<float><<<blocks, 256, 0, s>>>(a, part, slices, n, static_cast<float*>(dw));
  return hipGetLastError();
}

hipError_t launch_lm_terms(const float* in, int ld_in, const int* idx, const int* count, int rows, int cols, void* out,
                           hipStream_t s) {
  lm_terms_kernel<<<dim3(rows, (cols + 2047) / 2048), 256, 0, s>>>(in, ld_in, idx, count, cols,
                                                                   static_cast<size_t>(rows) * cols, static_cast<bf16_t*>(out));
  return hipGetLastError();
}

hipError_t launch_lm_head(int dtype, const void* w, int vocab, int d, void* w_t, int pitch, hipStream_t s) {
  const dim3 grid(d / 64, pitch / 64);
  if (dtype == 1)
    lm_head_kernel<bf16_t><<<grid, 256, 0, s>>>(static_cast<const bf16_t*>(w), vocab, d, static_cast<bf16_t*>(w_t), pitch);
  else
    lm_head_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(w), vocab, d, static_cast<float*>(w_t), pitch);
  return hipGetLastError();
}

}  // namespace hero
