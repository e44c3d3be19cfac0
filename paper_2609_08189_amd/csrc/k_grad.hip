// The global norm of many gradient tensors, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / norm)
//
// The tensors are one list of chunks; a workgroup takes a contiguous run of them, so that the
// sizes of the tensors do not matter (a model's router has tensors of 6 x 64 beside adapters of
// millions).  Squares are added in 64 bits: no gradient is too large or too small for its square,
// and the matrix pipes are idle anyway.  Each workgroup writes one partial sum; the pass that scales
// adds them again in every workgroup, in the same order, which saves a launch and a round trip.
// Nothing is added by atomics: the result does not depend on timing.  HBM bounds it: each gradient
// is read once for the norm, and read and written once to be scaled.
#include <algorithm>

#include "hero_device.h"
#include "hero_kernels.h"

namespace hero {
namespace {

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[4];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (red[0] + red[1]) + (red[2] + red[3]);
  __syncthreads();
  return v;
}

// the tensor that chunk c belongs to (chunk0 ascending, tensors without chunks skipped)
__device__ __forceinline__ int tensor_of(const GradTable& tab, uint32_t c) {
  int lo = 0, hi = tab.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (tab.chunk0[mid] <= c)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// f(chunk's first element, its elements, tensor) for the chunks of workgroup b
template <class F>
__device__ __forceinline__ void for_chunks(const GradTable& tab, uint32_t b, F f) {
  const uint64_t total = tab.chunk0[tab.n];
  uint32_t c = static_cast<uint32_t>(total * b / gridDim.x);
  const uint32_t end = static_cast<uint32_t>(total * (b + 1) / gridDim.x);
  if (c >= end) return;
  int i = tensor_of(tab, c);
  for (; c < end; ++c) {
    while (tab.chunk0[i + 1] <= c) ++i;
    const size_t at = static_cast<size_t>(c - tab.chunk0[i]) * kGradChunk;
    f(at, static_cast<int>(min(static_cast<size_t>(kGradChunk), static_cast<size_t>(tab.count[i]) - at)), i);
  }
}

// 16 bytes of a tensor per lane
template <typename T> struct Vec;
template <> struct Vec<float> { static constexpr int N = 4; };
template <> struct Vec<bf16_t> { static constexpr int N = 8; };

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* __restrict__ g, int n) {
  constexpr int N = Vec<T>::N;
  double s[N];
#pragma unroll
  for (int k = 0; k < N; ++k) s[k] = 0.0;
  const int nv = (reinterpret_cast<uintptr_t>(g) & 15u) == 0 ? n / N : 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += 256) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(g + static_cast<size_t>(i) * N);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (N == 4) {
        const double x = static_cast<double>(__uint_as_float(v[k]));
        s[k] = fma(x, x, s[k]);
      } else {
        const double x = static_cast<double>(__uint_as_float(v[k] << 16));
        const double y = static_cast<double>(__uint_as_float(v[k] & 0xffff0000u));
        s[2 * k] = fma(x, x, s[2 * k]);
        s[2 * k + 1] = fma(y, y, s[2 * k + 1]);
      }
    }
  }
  for (int i = nv * N + threadIdx.x; i < n; i += 256) {
    const double x = static_cast<double>(ldf(g + i));
    s[0] = fma(x, x, s[0]);
  }
  double v = 0.0;
#pragma unroll
  for (int k = 0; k < N; ++k) v += s[k];
  return v;
}

// o = g (pre c): pre is a power of two, so that c is a normal number however small the factor
template <typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* o, int n, float pre, float c) {
  constexpr int N = Vec<T>::N;
  const int nv = ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(o)) & 15u) == 0 ? n / N : 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < nv; i += 256) {
    u32x4 v = *reinterpret_cast<const u32x4*>(g + static_cast<size_t>(i) * N);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (N == 4) {
        v[k] = __float_as_uint(__uint_as_float(v[k]) * pre * c);
      } else {
        const bf16_t lo = f32_to_bf16(__uint_as_float(v[k] << 16) * pre * c);
        const bf16_t hi = f32_to_bf16(__uint_as_float(v[k] & 0xffff0000u) * pre * c);
        v[k] = static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
      }
    }
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(o + static_cast<size_t>(i) * N));
  }
  for (int i = nv * N + threadIdx.x; i < n; i += 256) stf(o + i, ldf(g + i) * pre * c);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(GradTable tab, double* __restrict__ part) {
  double s = 0.0;
  for_chunks(tab, blockIdx.x, [&](size_t at, int n, int i) {
    if (tab.bf16[i])
      s += chunk_squares(static_cast<const bf16_t*>(tab.grad[i]) + at, n);
    else
      s += chunk_squares(static_cast<const float*>(tab.grad[i]) + at, n);
  });
  s = block_sum(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double* __restrict__ part, int n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += part[i];
  return sqrt(block_sum(s));
}

__global__ __launch_bounds__(256) void grad_norm_finish(const double* __restrict__ part, int n,
                                                        float* __restrict__ norm) {
  const double v = norm_of(part, n);
  if (threadIdx.x == 0) *norm = static_cast<float>(v);
}

__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable tab, const double* __restrict__ part, int n,
                                                        double max_norm, float* __restrict__ norm) {
  const double v = norm_of(part, n);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(v);
  // a norm that is not a number makes every gradient one, an infinite one leaves zeros and NaN
  const double f = v <= max_norm ? 1.0 : max_norm / v;
  const float pre = f < 0x1p-64 ? 0x1p-64f : 1.0f, c = static_cast<float>(f < 0x1p-64 ? f * 0x1p64 : f);
  // from the last chunk to the first: what the norm read last is still in the last-level cache
  for_chunks(tab, gridDim.x - 1 - blockIdx.x, [&](size_t at, int m, int i) {
    if (pre * c == 1.0f && tab.grad[i] == tab.out[i]) return;   // in place and unchanged
    if (tab.bf16[i])
      chunk_scale(static_cast<const bf16_t*>(tab.grad[i]) + at, static_cast<bf16_t*>(tab.out[i]) + at, m, pre, c);
    else
      chunk_scale(static_cast<const float*>(tab.grad[i]) + at, static_cast<float*>(tab.out[i]) + at, m, pre, c);
  });
}

}  // namespace

hipError_t launch_grad_norm(const GradTable& tab, int groups, double* part, hipStream_t s) {
  grad_norm_kernel<<<groups, 256, 0, s>>>(tab, part);
  return hipGetLastError();
}

hipError_t launch_grad_norm_finish(const double* part, int n, float* norm, hipStream_t s) {
  grad_norm_finish<<<1, 256, 0, s>>>(part, n, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradTable& tab, int groups, const double* part, int n, float max_norm, float* norm,
                            hipStream_t s) {
  grad_clip_kernel<<<groups, 256, 0, s>>>(tab, part, n, static_cast<double>(max_norm), norm);
  return hipGetLastError();
}

}  // namespace hero
