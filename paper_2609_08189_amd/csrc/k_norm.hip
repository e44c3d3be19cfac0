// The final RMSNorm of the model, between the stack's output and the LM head, and its backward.
//
//   x  = h r w,                      r = (mean h^2 + eps)^(-1/2)
//   dh = r u - h r^3 <h, u> / d,     u = w dx
//   dw = sum over the rows of dx h r
//
// A row is read once into registers, by one wave (many rows) or by the four waves of a workgroup (few rows,
// wide rows); sums are fp32, every output is rounded once.  HBM bounds both: 2 accesses an element forwards,
// 3 backwards.  The backward's workgroups keep the gain's gradient of their rows in registers and write one
// partial row each; a second launch adds those in order, so the result does not depend on timing.
#include <algorithm>

#include "hero_device.h"
#include "hero_kernels.h"

namespace hero {
namespace {

constexpr int kNormThreads = 256;
constexpr int kWideRow = 8192;      // widest row of one wave: 16 chunks of eight elements a lane
constexpr int kGainGroups = 512;    // workgroups of a backward with the gain's gradient

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
  extern __shared__ float gsum[];   // GAIN, one wave a row: d floats
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
  for (int t = first; t < rows; t += step) {
    const size_t at = static_cast<size_t>(t) * d;
    Raw8<T> v[NC], y[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (lane + i * L < nc) {
        v[i].load(h + at + 8 * (lane + i * L));
        y[i].load(dx + at + 8 * (lane + i * L));
      }
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
  }
  if constexpr (GAIN) {
    float* out = part + static_cast<size_t>(blockIdx.x) * d;
    if constexpr (WPR == 4) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (lane + i * L < nc) st8(out + 8 * (lane + i * L), acc[i]);
    } else {
      for (int q = 0; q < 4; ++q) {   // the four waves' rows, added in order
        if (wave == q)
#pragma unroll
          for (int i = 0; i < NC; ++i)
            if (lane + i * L < nc)
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                float* p = gsum + 8 * (lane + i * L) + k;
                *p = q ? *p + acc[i][k] : acc[i][k];
              }
        __syncthreads();
      }
      for (int i = threadIdx.x; i < d; i += kNormThreads) out[i] = gsum[i];
    }
  }
}

// out[i] = sum over the groups of part[g][i], 64 columns a workgroup, its four waves a quarter of the groups each
__global__ __launch_bounds__(256) void gain_reduce_kernel(const float* __restrict__ part, int groups, int d,
                                                          float* __restrict__ out) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  const int per = (groups + 3) / 4, g1 = min(groups, (wave + 1) * per);
  if (i < d) {
    int g = wave * per;
    for (; g + 4 <= g1; g += 4)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += part[static_cast<size_t>(g + k) * d + i];
    for (; g < g1; ++g) s[0] += part[static_cast<size_t>(g) * d + i];
  }
  red[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (wave == 0 && i < d) out[i] = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

// chunks of eight elements a lane holds: the smallest compiled count that covers the row
int norm_chunks(int d, int wpr) { return (d / 8 + 64 * wpr - 1) / (64 * wpr); }

// Few rows leave CUs idle with a wave a row, and a wave's chain of loads is four times as long as a
// workgroup's: a row takes a whole workgroup then, and where it is wider than a wave's registers.
bool norm_whole_group(int T, int d) { return T <= 4 * 256 || d > kWideRow; }

template <typename T>
hipError_t norm_fwd(const void* h, const void* w, int rows, int d, float eps, void* x, hipStream_t s) {
  const T *hh = static_cast<const T*>(h), *ww = static_cast<const T*>(w);
  T* xx = static_cast<T*>(x);
#define HERO_NORM(NC, WPR) \
  final_norm_kernel<T, NC, WPR><<<WPR == 4 ? rows : (rows + 3) / 4, kNormThreads, 0, s>>>(hh, ww, rows, d, eps, xx)
  if (norm_whole_group(rows, d)) {
    const int n = norm_chunks(d, 4);
    if (n <= 1) HERO_NORM(1, 4);
    else if (n <= 2) HERO_NORM(2, 4);
    else if (n <= 4) HERO_NORM(4, 4);
    else HERO_NORM(16, 4);
  } else {
    const int n = norm_chunks(d, 1);
    if (n <= 2) HERO_NORM(2, 1);
    else if (n <= 4) HERO_NORM(4, 1);
    else if (n <= 8) HERO_NORM(8, 1);
    else if (n <= 10) HERO_NORM(10, 1);
    else HERO_NORM(16, 1);
  }
#undef HERO_NORM
  return hipGetLastError();
}

template <typename T, bool GAIN>
hipError_t norm_bwd(const void* h, const void* dx, const void* w, int rows, int d, float eps, void* dh, float* part,
                    hipStream_t s) {
  const T *hh = static_cast<const T*>(h), *yy = static_cast<const T*>(dx), *ww = static_cast<const T*>(w);
  T* oo = static_cast<T*>(dh);
#define HERO_NORM(NC, WPR)                                                                                    \
  final_norm_bwd_kernel<T, NC, WPR, GAIN>                                                                     \
      <<<GAIN ? final_norm_bwd_groups(rows, d) : WPR == 4 ? rows : (rows + 3) / 4, kNormThreads,              \
         GAIN && WPR == 1 ? d * 4 : 0, s>>>(hh, yy, ww, rows, d, eps, oo, part)
  if (norm_whole_group(rows, d)) {
    const int n = norm_chunks(d, 4);
    if (n <= 1) HERO_NORM(1, 4);
    else if (n <= 2) HERO_NORM(2, 4);
    else if (n <= 4) HERO_NORM(4, 4);
    else HERO_NORM(16, 4);
  } else {
    const int n = norm_chunks(d, 1);
    if (n <= 2) HERO_NORM(2, 1);
    else if (n <= 4) HERO_NORM(4, 1);
    else if (n <= 8) HERO_NORM(8, 1);
    else if (n <= 10) HERO_NORM(10, 1);
    else HERO_NORM(16, 1);
  }
#undef HERO_NORM
  return hipGetLastError();
}

}  // namespace

int final_norm_bwd_groups(int T, int d) {
  return std::min(norm_whole_group(T, d) ? T : (T + 3) / 4, kGainGroups);
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
  gain_reduce_kernel<<<(d + 63) / 64, 256, 0, s>>>(part, final_norm_bwd_groups(T, d), d, dnorm_w);
  return hipGetLastError();
}

}  // namespace hero
