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
// than e^60 above its target changes its reference on the way (EpiLmExp, lm_combine_kernel).
//
// Tokens without a target cost nothing: the rows that count are compacted on the device, and every product
// takes their number from there.  The passes here are a row or a token a wave and read what the products
// left in the last-level cache; the products (k_gemm.hip) bound the whole.
#include <limits.h>

#include <algorithm>

#include "hero_device.h"
#include "hero_kernels.h"

namespace hero {
namespace {

constexpr int kRowsThreads = 1024;

// Ordered compaction by one workgroup, a run of neighbouring tokens per thread.
__global__ __launch_bounds__(kRowsThreads) void lm_rows_kernel(LmRows a, int chunk, int n_chunks) {
  __shared__ int wsum[kRowsThreads / kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (a.T + kRowsThreads - 1) / kRowsThreads;
  const int t0 = min(a.T, static_cast<int>(threadIdx.x) * per), t1 = min(a.T, t0 + per);
  int n = 0;
  for (int t = t0; t < t1; ++t) n += static_cast<unsigned>(a.targets[t]) < static_cast<unsigned>(a.vocab);
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
  for (int t = t0; t < t1; ++t) {
    const bool in = static_cast<unsigned>(a.targets[t]) < static_cast<unsigned>(a.vocab);
    a.inv[t] = in ? m : -1;
    if (in) a.idx[m++] = t;
  }
  for (int i = total + threadIdx.x; i < a.T; i += kRowsThreads) a.idx[i] = 0;   // rows that no result uses
  if (threadIdx.x == 0) a.counts[0] = total;
  for (int c = threadIdx.x; c < n_chunks; c += kRowsThreads) a.counts[1 + c] = max(0, min(chunk, total - c * chunk));
}

// The target's logit, a wave a row
template <typename T>
__global__ __launch_bounds__(256) void lm_targets_kernel(LmRows a) {
  const int lane = threadIdx.x & 63, m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= a.counts[0]) return;
  const int t = a.idx[m], y = a.targets[t];
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

// The sums of a row's pieces of 64 columns, a wave a row.  A piece whose reference is not the row's (a logit
// far above the target's) raises the row's: then the earlier sums, and this piece's e, are rescaled.
__global__ __launch_bounds__(256) void lm_combine_kernel(LmRows a, LmPiece p, int parts) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), m = p.m0 + i;
  if (i >= *p.count) return;
  const float r0 = a.ref[m];
  const float2* part = p.part + static_cast<size_t>(i) * parts;
  float s = 0.f, r = r0;
  for (int q = lane; q < parts; q += kWave) r = fmaxf(r, part[q].x);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) r = fmaxf(r, __shfl_xor(r, off, kWave));
  const bool raised = r > r0;
  for (int q = lane; q < parts; q += kWave) {
    const float2 v = part[q];
    s += raised ? v.y * __expf(v.x - r) : v.y;
  }
  s = wave_sum(s);
  const float f0 = raised ? __expf(r0 - r) : 1.0f;
  if (lane == 0) {
    a.sum[m] = fmaf(a.sum[m], f0, s);
    a.alpha[m] = f0;
    a.ref[m] = r;
  }
  if (!raised || !p.e) return;
  bf16_t* e = static_cast<bf16_t*>(p.e) + static_cast<size_t>(i) * p.pitch;
  for (int n = lane; n < p.pitch; n += kWave) {   // the columns of wave q of tile n / 256: (n & 127) / 32
    const float f = __expf(part[(n >> 8) * 4 + ((n & 127) >> 5)].x - r);
    e[n] = f32_to_bf16(bf16_to_f32(e[n]) * f);
  }
}

// fp32: the logits of a piece to e, in place, a workgroup a row; with zeros up to the pitch
__global__ __launch_bounds__(256) void lm_exp_f32_kernel(LmRows a, LmPiece p) {
  __shared__ float red[4];
  const int i = blockIdx.x, m = p.m0 + i, wave = threadIdx.x >> 6;
  if (i >= *p.count) return;
  const float r0 = a.ref[m];
  const int tgt = a.tgt[m] - p.v0;
  float* e = static_cast<float*>(p.e) + static_cast<size_t>(i) * p.pitch;
  float r = r0;
  for (int n = threadIdx.x; n < p.cols; n += 256) r = fmaxf(r, e[n]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) r = fmaxf(r, __shfl_xor(r, off, kWave));
  if ((threadIdx.x & 63) == 0) red[wave] = r;
  __syncthreads();
  r = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  __syncthreads();
  // the target's logit is a good reference unless the row rises far above it
  if (!(r - r0 > 60.0f)) r = r0;
  float s = 0.f;
  for (int n = threadIdx.x; n < p.pitch; n += 256) {
    const float v = n < p.cols && n != tgt ? expf(e[n] - r) : 0.f;
    e[n] = v;
    s += v;
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    const float f0 = r > r0 ? expf(r0 - r) : 1.0f;
    a.sum[m] = fmaf(a.sum[m], f0, (red[0] + red[1]) + (red[2] + red[3]));
    a.alpha[m] = f0;
    a.ref[m] = r;
  }
}

// log(1 + S) from S = sum e^(lt - ref) ...: the row's sum is in units of its reference
__device__ __forceinline__ float row_nll(float lt, float ref, float s) {
  return lt == ref ? log1pf(s) : logf(s + expf(lt - ref)) + (ref - lt);
}

// A token a wave, for the tokens whose row is in the chunk; workgroup 0 of the last chunk adds the loss.
template <typename T>
__global__ __launch_bounds__(256) void lm_finish_kernel(LmRows a, LmFinish f) {
  const int lane = threadIdx.x & 63, N = a.counts[0];
  if (blockIdx.x == 0) {
    if (!f.last) return;
    __shared__ double red[256];
    double s = 0.0;
    for (int m = threadIdx.x; m < N; m += 256) s += static_cast<double>(row_nll(a.lt[m], a.ref[m], a.sum[m]));
    red[threadIdx.x] = s;
    __syncthreads();
    for (int k = 128; k > 0; k >>= 1) {
      if (static_cast<int>(threadIdx.x) < k) red[threadIdx.x] += red[threadIdx.x + k];
      __syncthreads();
    }
    if (threadIdx.x == 0) f.loss[0] = static_cast<float>(f.scale * (f.mean ? red[0] / max(N, 1) : red[0]));
    return;
  }
  const int t = (blockIdx.x - 1) * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const int m = a.inv[t];
  if (m < 0) {
    if (!f.last) return;
    if (lane == 0 && f.token_loss) f.token_loss[t] = 0.f;
    if (f.dx) {
      const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      for (int c = lane; c < a.d / 8; c += kWave) st8(static_cast<T*>(f.dx) + static_cast<size_t>(t) * a.d + 8 * c, z);
    }
    return;
  }
  if (m < f.m0 || m >= f.m0 + f.chunk) return;
  const float lt = a.lt[m], ref = a.ref[m], s = a.sum[m], z = s + (lt == ref ? 1.0f : expf(lt - ref));
  const float unit = f.mean ? f.scale / static_cast<float>(N) : f.scale;
  if (lane == 0) {
    const float nll = row_nll(lt, ref, s);
    if (f.token_loss) f.token_loss[t] = nll;
    if (f.lse) {
      f.lse[m] = lt + nll;
      f.own[m] = -s / z;
    }
  }
  if (!f.dx) return;
  const T* w = static_cast<const T*>(a.w) + static_cast<size_t>(a.tgt[m]) * a.d;
  const float* acc = f.acc + static_cast<size_t>(m - f.m0) * a.d;
  const size_t stride = static_cast<size_t>(f.chunk) * a.d;
  const float inv = 1.0f / z;
  for (int c = lane; c < a.d / 8; c += kWave) {
    float o[8];
    Raw8<T> wv;
    wv.load(w + 8 * c);
    Raw8<float> v;
    v.load(acc + 8 * c);
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = v[k];
    for (int q = 1; q < f.slices; ++q) {
      v.load(acc + q * stride + 8 * c);
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] += v[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = unit * ((o[k] - s * wv[k]) * inv);
    st8(static_cast<T*>(f.dx) + static_cast<size_t>(t) * a.d + 8 * c, o);
  }
}

// xT[i][m] = x[idx[m]][i], zero for m at or past the counted rows; 64 x 64 tiles
template <typename T>
__global__ __launch_bounds__(256) void lm_xT_kernel(LmRows a, T* __restrict__ xT, int pitch) {
  __shared__ T tile[64][65];
  const int N = a.counts[0], i0 = blockIdx.x * 64, m0 = blockIdx.y * 64;
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  for (int k = ty; k < 64; k += 4) {
    const int m = m0 + k;
    tile[k][tx] = m < N ? static_cast<const T*>(a.x)[static_cast<size_t>(a.idx[m]) * a.d + i0 + tx] : T(0);
  }
  __syncthreads();
  for (int k = ty; k < 64; k += 4) xT[static_cast<size_t>(i0 + k) * pitch + m0 + tx] = tile[tx][k];
}

// fp32: g[v][m] = unit (p - [target]) from the logits [rows][ldl], transposed
__global__ __launch_bounds__(256) void lm_g_f32_kernel(LmRows a, int v0, int cols, const float* __restrict__ lse,
                                                       const float* __restrict__ own, const float* __restrict__ logits,
                                                       int ldl, float scale, int mean, float* __restrict__ g,
                                                       int pitch) {
  __shared__ float tile[64][65];
  const int N = a.counts[0], n0 = blockIdx.x * 64, m0 = blockIdx.y * 64;
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const float unit = mean ? scale / static_cast<float>(max(N, 1)) : scale;
  for (int k = ty; k < 64; k += 4) {
    const int m = m0 + k, n = n0 + tx;
    float v = 0.f;
    if (m < N && n < cols)
      v = unit * (a.tgt[m] == v0 + n ? own[m] : expf(logits[static_cast<size_t>(m) * ldl + n] - lse[m]));
    tile[k][tx] = v;
  }
  __syncthreads();
  for (int k = ty; k < 64; k += 4)
    if (n0 + k < cols) g[static_cast<size_t>(n0 + k) * pitch + m0 + tx] = tile[tx][k];
}

}  // namespace

hipError_t launch_lm_rows(const LmRows& a, int chunk, int n_chunks, hipStream_t s) {
  lm_rows_kernel<<<1, kRowsThreads, 0, s>>>(a, chunk, n_chunks);
  return hipGetLastError();
}

hipError_t launch_lm_targets(const LmRows& a, hipStream_t s) {
  if (a.dtype == 1)
    lm_targets_kernel<bf16_t><<<(a.T + 3) / 4, 256, 0, s>>>(a);
  else
    lm_targets_kernel<float><<<(a.T + 3) / 4, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_combine(const LmRows& a, const LmPiece& p, hipStream_t s) {
  if (a.dtype == 1)
    lm_combine_kernel<<<(p.rows_max + 3) / 4, 256, 0, s>>>(a, p, lm_parts(p.cols));
  else
    lm_exp_f32_kernel<<<p.rows_max, 256, 0, s>>>(a, p);
  return hipGetLastError();
}

hipError_t launch_lm_finish(const LmRows& a, const LmFinish& f, hipStream_t s) {
  if (a.dtype == 1)
    lm_finish_kernel<bf16_t><<<1 + (a.T + 3) / 4, 256, 0, s>>>(a, f);
  else
    lm_finish_kernel<float><<<1 + (a.T + 3) / 4, 256, 0, s>>>(a, f);
  return hipGetLastError();
}

hipError_t launch_lm_xT(const LmRows& a, void* xT, int pitch, hipStream_t s) {
  const dim3 grid(a.d / 64, pitch / 64);
  if (a.dtype == 1)
    lm_xT_kernel<bf16_t><<<grid, 256, 0, s>>>(a, static_cast<bf16_t*>(xT), pitch);
  else
    lm_xT_kernel<float><<<grid, 256, 0, s>>>(a, static_cast<float*>(xT), pitch);
  return hipGetLastError();
}

hipError_t launch_lm_g_f32(const LmRows& a, int v0, int cols, const float* lse, const float* own, const float* logits,
                           int ldl, float scale, bool mean, float* g, int pitch, hipStream_t s) {
  lm_g_f32_kernel<<<dim3((cols + 63) / 64, pitch / 64), 256, 0, s>>>(a, v0, cols, lse, own, logits, ldl, scale,
                                                                     mean ? 1 : 0, g, pitch);
  return hipGetLastError();
}

}  // namespace hero
