// The final RMSNorm of the model, between the stack's output and the LM head, and its backward.
//
//   x  = h r w,                      r = (mean h^2 + eps)^(-1/2)
//   dh = r u - h r^3 <h, u> / d,     u = w dx
//   dw = sum over the rows of dx h r
//
// A row is read once into registers, by one wave (narrow rows) or by the four waves of a workgroup; sums are
// fp32, every output is rounded once.  HBM bounds both: 2 accesses an element forwards, 3 backwards.  For the
// gain's gradient a workgroup (or wave) takes several rows, the next one's loads under way, keeps their sum in
// registers and writes one partial row; a second launch adds those in order, so the result does not depend on timing.
#include <algorithm>
#include <type_traits>

#include "hero_device.h"
#include "hero_kernels.h"

namespace hero {
namespace {

constexpr int kNormThreads = 256;
// Most partial rows of the gain's gradient: a workgroup each (8192 x 5120: 512, 1024, 2048 of them 74, 66, 78 us) or a
// wave (30000 x 512: 63, 36, 28).
constexpr int kGainRows = 1024, kGainWaveRows = 2048;
// A wave a row up to here: with a workgroup a row half of its threads or more would have nothing to do.  The
// width alone decides, so that a row's sums have one order whatever the call.
constexpr int kWaveRow = 1024;

// sum over a row's WPR waves (a workgroup's, if more than one), left in every lane
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float (&red)[2][4], int& turn) {
  v = wave_sum(v);
  if constexpr (WPR == 4) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) red[turn][w] = v;
    __syncthreads();
    v = (red[turn][0] + red[turn][1]) + (red[turn][2] + red[turn][3]);
    turn ^= 1;   // the next sum writes the other set: no second barrier
  }
  return v;
}

template <typename T, int NC, int WPR>
__global__ __launch_bounds__(kNormThreads) void final_norm_kernel(const T* __restrict__ h, const T* __restrict__ w,
                                                                  int rows, int d, float eps, T* __restrict__ x) {
  __shared__ float red[2][4];
  int turn = 0;
  constexpr int L = 64 * WPR;
  const int lane = WPR == 4 ? threadIdx.x : threadIdx.x & 63;
  const int t = WPR == 4 ? blockIdx.x : blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= rows) return;
  const T* row = h + static_cast<size_t>(t) * d;
  const int nc = d >> 3;
  Raw8<T> v[NC], g[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (lane + i * L < nc) {
      v[i].load(row + 8 * (lane + i * L));
      g[i].load(w + 8 * (lane + i * L));
    }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (lane + i * L < nc)
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(v[i][k], v[i][k], ss);
  ss = row_sum<WPR>(ss, red, turn);
  const float r = 1.0f / sqrtf(ss / static_cast<float>(d) + eps);
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (lane + i * L < nc) {
      float o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = v[i][k] * r * g[i][k];
      st8(x + static_cast<size_t>(t) * d + 8 * (lane + i * L), o);
    }
}

template <typename T, int NC, int WPR, bool GAIN>
__global__ __launch_bounds__(kNormThreads) void final_norm_bwd_kernel(const T* __restrict__ h, const T* __restrict__ dx,
                                                                      const T* __restrict__ w, int rows, int d,
                                                                      float eps, T* __restrict__ dh,
                                                                      float* __restrict__ part) {
  __shared__ float red[2][4];
  int turn = 0;
  constexpr int L = 64 * WPR;
  const int lane = WPR == 4 ? threadIdx.x : threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nc = d >> 3;
  const int first = WPR == 4 ? blockIdx.x : blockIdx.x * 4 + wave, step = WPR == 4 ? gridDim.x : gridDim.x * 4;
  float acc[GAIN ? NC : 1][8];
  if constexpr (GAIN)
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[i][k] = 0.f;
  Raw8<T> v[NC], y[NC], nv[NC], ny[NC];
  auto fetch = [&](Raw8<T>(&a)[NC], Raw8<T>(&b)[NC], int t) {
    const size_t at = static_cast<size_t>(t) * d;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (lane + i * L < nc) {
        a[i].load(h + at + 8 * (lane + i * L));
        b[i].load(dx + at + 8 * (lane + i * L));
      }
  };
  if (first < rows) fetch(v, y, first);
  for (int t = first; t < rows; t += step) {
    const size_t at = static_cast<size_t>(t) * d;
    if constexpr (GAIN)   // several rows a workgroup: the next one's loads are under way
      if (t + step < rows) fetch(nv, ny, t + step);
    float ss = 0.f, hu = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (lane + i * L < nc) {
        Raw8<T> g;
        g.load(w + 8 * (lane + i * L));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          ss = fmaf(v[i][k], v[i][k], ss);
          hu = fmaf(v[i][k], y[i][k] * g[k], hu);
        }
      }
    ss = row_sum<WPR>(ss, red, turn);
    hu = row_sum<WPR>(hu, red, turn);
    const float r = 1.0f / sqrtf(ss / static_cast<float>(d) + eps);
    const float c = r * r * (hu / static_cast<float>(d));
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (lane + i * L < nc) {
        Raw8<T> g;
        g.load(w + 8 * (lane + i * L));
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          o[k] = r * (y[i][k] * g[k] - v[i][k] * c);
          if constexpr (GAIN) acc[i][k] = fmaf(y[i][k], v[i][k] * r, acc[i][k]);
        }
        st8(dh + at + 8 * (lane + i * L), o);
      }
    if constexpr (GAIN)
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        v[i] = nv[i];
        y[i] = ny[i];
      }
  }
  if constexpr (GAIN) {
    float* out = part + static_cast<size_t>(first) * d;
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (lane + i * L < nc) st8(out + 8 * (lane + i * L), acc[i]);
  }
}

// out[i] = sum over the partial rows: 32 columns (a whole line) a workgroup, every 32nd row a thread, so that few
// rows of few columns still are many loads at once (1024 rows of 1024 columns, 64 columns a workgroup of four waves: 15 us)
__global__ __launch_bounds__(1024) void gain_reduce_kernel(const float* __restrict__ part, int rows, int d,
                                                           float* __restrict__ out) {
  __shared__ float red[32][33];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5, i = blockIdx.x * 32 + c;
  float s = 0.f;
#pragma unroll 16
  for (int g = r; g < rows; g += 32) s += part[static_cast<size_t>(g) * d + i];
  red[r][c] = s;
  __syncthreads();
#pragma unroll
  for (int k = 16; k > 0; k >>= 1) {
    if (r < k) red[r][c] += red[r + k][c];
    __syncthreads();
  }
  if (r == 0) out[i] = red[0][c];
}

// f(chunks of eight elements a lane holds, waves a row): the smallest compiled count that covers the row
template <class F>
void norm_shape(int d, F f) {
  const int n = (d / 8 + 255) / 256;
  if (d <= 512) f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  else if (d <= kWaveRow) f(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
  else if (n <= 1) f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
  else if (n <= 2) f(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
  else if (n <= 3) f(std::integral_constant<int, 3>(), std::integral_constant<int, 4>());
  else if (n <= 4) f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
  else f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
}

template <typename T>
hipError_t norm_fwd(const void* h, const void* w, int rows, int d, float eps, void* x, hipStream_t s) {
  norm_shape(d, [&](auto nc, auto wpr) {
    constexpr int NC = decltype(nc)::value, WPR = decltype(wpr)::value;
    final_norm_kernel<T, NC, WPR><<<WPR == 4 ? rows : (rows + 3) / 4, kNormThreads, 0, s>>>(
        static_cast<const T*>(h), static_cast<const T*>(w), rows, d, eps, static_cast<T*>(x));
  });
  return hipGetLastError();
}

template <typename T, bool GAIN>
hipError_t norm_bwd(const void* h, const void* dx, const void* w, int rows, int d, float eps, void* dh, float* part,
                    hipStream_t s) {
  norm_shape(d, [&](auto nc, auto wpr) {
    constexpr int NC = decltype(nc)::value, WPR = decltype(wpr)::value;
    const int n = GAIN ? final_norm_bwd_groups(rows, d) : rows;
    final_norm_bwd_kernel<T, NC, WPR, GAIN><<<WPR == 4 ? n : (n + 3) / 4, kNormThreads, 0, s>>>(
        static_cast<const T*>(h), static_cast<const T*>(dx), static_cast<const T*>(w), rows, d, eps, static_cast<T*>(dh),
        part);
  });
  return hipGetLastError();
}

}  // namespace

// partial rows: a workgroup's or a wave's each, whole workgroups
int final_norm_bwd_groups(int T, int d) {
  return (std::min(T, d <= kWaveRow ? kGainWaveRows : kGainRows) + 3) / 4 * 4;
}

hipError_t launch_final_norm(int dtype, const void* h, const void* norm_w, int T, int d, float eps, void* x,
                             hipStream_t s) {
  return dtype == 1 ? norm_fwd<bf16_t>(h, norm_w, T, d, eps, x, s) : norm_fwd<float>(h, norm_w, T, d, eps, x, s);
}

hipError_t launch_final_norm_bwd(int dtype, const void* h, const void* dx, const void* norm_w, int T, int d, float eps,
                                 void* dh, float* dnorm_w, float* part, hipStream_t s) {
  hipError_t e;
  if (dtype == 1)
    e = dnorm_w ? norm_bwd<bf16_t, true>(h, dx, norm_w, T, d, eps, dh, part, s)
                : norm_bwd<bf16_t, false>(h, dx, norm_w, T, d, eps, dh, part, s);
  else
    e = dnorm_w ? norm_bwd<float, true>(h, dx, norm_w, T, d, eps, dh, part, s)
                : norm_bwd<float, false>(h, dx, norm_w, T, d, eps, dh, part, s);
  if (e != hipSuccess || !dnorm_w) return e;
  gain_reduce_kernel<<<d / 32, 1024, 0, s>>>(part, final_norm_bwd_groups(T, d), d, dnorm_w);
  return hipGetLastError();
}

}  // namespace hero
