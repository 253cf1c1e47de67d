// Layer norm of the MoE block's input rows (moe_layer_norm, moe_layer_norm_bwd):
//   s = round(x + residual),  mu = mean_c s,  rstd = (mean_c (s - mu)^2 + eps)^-1/2
//   y = round((s - mu) rstd gamma + beta)
// and, with xh = (s - mu) rstd and g = gamma dy,
//   dx = round(rstd (g - mean_c g - xh mean_c (g xh)) + dres)
//   dgamma = sum_t dy xh,  dbeta = sum_t dy
// All are HBM-bound.  The variance is the mean of the centred squares (a second
// pass over the row), so a large common offset costs no digits.
#include "common.hpp"
#include "internal.hpp"

namespace laep {
namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWaves = kNormThreads / kWave;

// Sum over the workgroup, the same bits in every thread (waves in order).
__device__ __forceinline__ float block_sum(float v, float* s_red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) s_red[threadIdx.x / kWave] = v;
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < kNormWaves; ++w) t += s_red[w];
  return t;
}

// the bits a value keeps in the row's storage type
template <typename T> __device__ __forceinline__ float stored(float v);
template <> __device__ __forceinline__ float stored<float>(float v) { return v; }
template <> __device__ __forceinline__ float stored<bf16_t>(float v) {
  return bf16_to_f32(f32_to_bf16(v));
}

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_kernel(
    const T* x, const T* residual, const float* __restrict__ gamma,
    const float* __restrict__ beta, int d, float eps, T* sum_out, T* __restrict__ y,
    float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_red[kNormWaves];
  const size_t row = (size_t)blockIdx.x * d;
  const int nvec = d / 8;
  auto load = [&](int v, float s[8]) {
    Elem<T>::load8(x + row + (size_t)v * 8, s);
    if (residual) {
      float r[8];
      Elem<T>::load8(residual + row + (size_t)v * 8, r);
#pragma unroll
      for (int q = 0; q < 8; ++q) s[q] = stored<T>(s[q] + r[q]);
    }
  };
  float sum = 0.0f;
  for (int v = threadIdx.x; v < nvec; v += kNormThreads) {
    float s[8];
    load(v, s);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum += s[q];
  }
  const float mu = block_sum(sum, s_red) / (float)d;
  float sq = 0.0f;
  for (int v = threadIdx.x; v < nvec; v += kNormThreads) {
    float s[8];
    load(v, s);
#pragma unroll
    for (int q = 0; q < 8; ++q) sq += (s[q] - mu) * (s[q] - mu);
  }
  const float rs = 1.0f / sqrtf(block_sum(sq, s_red) / (float)d + eps);
  for (int v = threadIdx.x; v < nvec; v += kNormThreads) {
    float s[8], g[8], o[8];
    load(v, s);
    if (sum_out) Elem<T>::store8(sum_out + row + (size_t)v * 8, s);
    Elem<float>::load8(gamma + (size_t)v * 8, g);
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (s[q] - mu) * rs * g[q];
    if (beta) {
      Elem<float>::load8(beta + (size_t)v * 8, g);
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] += g[q];
    }
    Elem<T>::store8(y + row + (size_t)v * 8, o);
  }
  if (threadIdx.x == 0) {
    if (mean) mean[blockIdx.x] = mu;
    if (rstd) rstd[blockIdx.x] = rs;
  }
}

// One workgroup per range of rows: dx of each, and the range's partial dgamma
// and dbeta rows, kept in LDS by the thread that owns the columns.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_kernel(
    const T* dy, const T* __restrict__ s, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, const T* dres, int n_rows,
    int rows_per, int d, T* dx, float* __restrict__ part) {
  __shared__ float s_red[kNormWaves];
  const int nvec = d / 8;
  const int r0 = blockIdx.x * rows_per, r1 = min(n_rows, r0 + rows_per);
  float* const pg = part ? part + (size_t)blockIdx.x * 2 * d : nullptr;
  for (int r = r0; r < r1; ++r) {
    const size_t row = (size_t)r * d;
    const float mu = mean[r], rs = rstd[r];
    float a = 0.0f, b = 0.0f;
    for (int v = threadIdx.x; v < nvec; v += kNormThreads) {
      float sv[8], dv[8], g[8];
      Elem<T>::load8(s + row + (size_t)v * 8, sv);
      Elem<T>::load8(dy + row + (size_t)v * 8, dv);
      Elem<float>::load8(gamma + (size_t)v * 8, g);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float xh = (sv[q] - mu) * rs;
        a += g[q] * dv[q];
        b += g[q] * dv[q] * xh;
      }
    }
    a = block_sum(a, s_red) / (float)d;
    b = block_sum(b, s_red) / (float)d;
    for (int v = threadIdx.x; v < nvec; v += kNormThreads) {
      float sv[8], dv[8], g[8], o[8];
      Elem<T>::load8(s + row + (size_t)v * 8, sv);
      Elem<T>::load8(dy + row + (size_t)v * 8, dv);
      Elem<float>::load8(gamma + (size_t)v * 8, g);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float xh = (sv[q] - mu) * rs;
        o[q] = rs * (g[q] * dv[q] - a - xh * b);
        sv[q] = dv[q] * xh;
      }
      if (dres) {
        Elem<T>::load8(dres + row + (size_t)v * 8, g);
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] += g[q];
      }
      Elem<T>::store8(dx + row + (size_t)v * 8, o);
      if (pg) {  // this thread's columns of the range's sums
        float* const w = pg + (size_t)v * 8;
        float* const bsum = w + d;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          w[q] = (r == r0 ? 0.0f : w[q]) + sv[q];
          bsum[q] = (r == r0 ? 0.0f : bsum[q]) + dv[q];
        }
      }
    }
  }
}

// dgamma, dbeta: the ranges' partial rows in order.
__global__ __launch_bounds__(256) void norm_bwd_reduce_kernel(const float* __restrict__ part,
                                                              int n_part, int d,
                                                              float* __restrict__ dgamma,
                                                              float* __restrict__ dbeta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= d) return;
  float g = 0.0f, b = 0.0f;
  for (int i = 0; i < n_part; ++i) {
    g += part[(size_t)i * 2 * d + c];
    b += part[(size_t)i * 2 * d + d + c];
  }
  dgamma[c] = g;
  if (dbeta) dbeta[c] = b;
}

constexpr int kNormParts = 512;

inline int norm_parts(int T) { return T < kNormParts ? T : kNormParts; }

}  // namespace

size_t layer_norm_bwd_ws_bytes(int T, int d) {
  return (size_t)norm_parts(T) * 2 * d * sizeof(float);
}

template <typename T>
static hipError_t norm_fwd_t(const T* x, const T* residual, const float* gamma, const float* beta,
                             int n, int d, float eps, T* sum_out, T* y, float* mean, float* rstd,
                             hipStream_t s) {
  hipLaunchKernelGGL(norm_fwd_kernel<T>, dim3((unsigned)n), dim3(kNormThreads), 0, s, x, residual,
                     gamma, beta, d, eps, sum_out, y, mean, rstd);
  return hipGetLastError();
}

hipError_t launch_layer_norm(const void* x, const void* residual, const float* gamma,
                             const float* beta, int dtype, int T, int d, float eps, void* sum_out,
                             void* y, float* mean, float* rstd, hipStream_t s) {
  if (dtype == kDtypeBf16)
    return norm_fwd_t(static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(residual), gamma,
                      beta, T, d, eps, static_cast<bf16_t*>(sum_out), static_cast<bf16_t*>(y),
                      mean, rstd, s);
  return norm_fwd_t(static_cast<const float*>(x), static_cast<const float*>(residual), gamma, beta,
                    T, d, eps, static_cast<float*>(sum_out), static_cast<float*>(y), mean, rstd,
                    s);
}

template <typename T>
static hipError_t norm_bwd_t(const T* dy, const T* sv, const float* gamma, const float* mean,
                             const float* rstd, const T* dres, int n, int d, T* dx, float* dgamma,
                             float* dbeta, float* part, hipStream_t s) {
  const int parts = norm_parts(n);
  const int per = parts ? (n + parts - 1) / parts : 1;
  const int grid = (n + per - 1) / per;
  if (grid > 0)
    hipLaunchKernelGGL(norm_bwd_kernel<T>, dim3((unsigned)grid), dim3(kNormThreads), 0, s, dy, sv,
                       gamma, mean, rstd, dres, n, per, d, dx, dgamma ? part : nullptr);
  if (dgamma)
    hipLaunchKernelGGL(norm_bwd_reduce_kernel, dim3((unsigned)((d + 255) / 256)), dim3(256), 0, s,
                       part, grid, d, dgamma, dbeta);
  return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const void* dy, const void* sv, const float* gamma,
                                 const float* mean, const float* rstd, const void* dres, int dtype,
                                 int T, int d, void* dx, float* dgamma, float* dbeta, void* ws,
                                 hipStream_t s) {
  float* const part = static_cast<float*>(ws);
  if (dtype == kDtypeBf16)
    return norm_bwd_t(static_cast<const bf16_t*>(dy), static_cast<const bf16_t*>(sv), gamma, mean,
                      rstd, static_cast<const bf16_t*>(dres), T, d, static_cast<bf16_t*>(dx),
                      dgamma, dbeta, part, s);
  return norm_bwd_t(static_cast<const float*>(dy), static_cast<const float*>(sv), gamma, mean,
                    rstd, static_cast<const float*>(dres), T, d, static_cast<float*>(dx), dgamma,
                    dbeta, part, s);
}

}  // namespace laep
