// Layer norm of the MoE block's input rows (moe_layer_norm, moe_layer_norm_bwd):
//   s = round(x + residual),  mu = mean_c s,  rstd = (mean_c (s - mu)^2 + eps)^-1/2
//   y = round((s - mu) rstd gamma + beta)
// and, with xh = (s - mu) rstd and g = gamma dy,
//   dx = round(rstd (g - mean_c g - xh mean_c (g xh)) + dres)
//   dgamma = sum_t dy xh,  dbeta = sum_t dy
// All are HBM-bound.
#include <type_traits>

#include "common.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace laep {
namespace {

// 16 bytes of consecutive elements in their storage format, N of them, so that the
// lanes of a wave read and write one contiguous run (8 float32 columns a lane, two loads
// 32 bytes apart, took 45 us instead of 40 for the backward of 4000 x 4096 float32)
template <typename T> struct Vec;
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  u32x4_t r;
  __device__ __forceinline__ void load(const bf16_t* p) {
    r = ld_stream(reinterpret_cast<const u32x4_t*>(p));
  }
  __device__ __forceinline__ void get(float v[N]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = lo_bf16(r[i]);
      v[2 * i + 1] = hi_bf16(r[i]);
    }
  }
  // v rounded to storage, and widened again
  __device__ __forceinline__ void put(float v[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    get(v);
  }
  __device__ __forceinline__ void store(bf16_t* p) const {
    st_stream(reinterpret_cast<u32x4_t*>(p), r);
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  f32x4_t r;
  __device__ __forceinline__ void load(const float* p) {
    r = ld_stream(reinterpret_cast<const f32x4_t*>(p));
  }
  __device__ __forceinline__ void get(float v[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i];
  }
  __device__ __forceinline__ void put(float v[N]) { r = f32x4_t{v[0], v[1], v[2], v[3]}; }
  __device__ __forceinline__ void store(float* p) const {
    st_stream(reinterpret_cast<f32x4_t*>(p), r);
  }
};
template <int N>
__device__ __forceinline__ void load_f32(const float* p, float v[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4_t r = *reinterpret_cast<const f32x4_t*>(p + i);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[i + q] = r[q];
  }
}

// A row belongs to NL lanes, lane l holding the 16-byte vectors l, l + NL, ... (VPL of
// them), so it is read once; a workgroup walks the rows, several side by side where they
// are short, gamma, beta and, backwards, its columns' sums staying in registers.  NL is a
// power of two inside a wave, then the whole waves that hold the row (pairs of waves past
// 512 lanes) up to 1024 lanes, and only past those a lane holds more than one vector: a
// power of two leaves lanes idle (29392 x 2240 bf16 with a residual 110 us on 512 lanes,
// 90 on 320), and two vectors a lane have fewer loads in flight (8192 x 5120 bf16 75 us
// on 512 lanes, 57 on 640).
// Every lane loads, those past the row or the rows the last one's bytes, which they do not
// use: with a branch round the loads the compiler cannot tell which are pending where the
// paths join, and waits for the stores as well (8192 x 5120 69 us for 57, 3000 x 10240 58
// for 49).
// The waves' parts of a row's sums are added by lanes of each wave, a part a lane: every
// lane reading all of them took 93 registers for 47 at 1024 lanes of bf16, and a CU's
// second workgroup (12000 x 7168 bf16 without a residual 89 us for 66).
// Forward with a residual: workgroups for about 19 waves a CU, each row's loads issued after
// the last one's stores: 181 us at 32768 x 4096 bf16 (5.9 TB/s of 6.2 that a copy
// reaches), 24 us at 8192 x 2048; loading the next row ahead 202 and 27, a workgroup for
// every row 205 and 26.  Without one a row has half the loads, and the next row's go
// ahead of this row's sums: 8192 x 2048 14.6 us for 15.1, 4000 x 5120 float32 34 for 41.
// Backward: 256 workgroups, since each writes a row of partial sums, of up to 1024
// threads, with the next row's loads ahead: 174 us (6.2 TB/s) at 32768 x 4096 bf16 with
// dres, 28 us at 8192 x 2048; 512 threads 179 and 29, two rows ahead 172 and 29 there but
// 78 against 74 at 30000 x 1000 float32; 512 workgroups 195 and 31.
constexpr int kFwdThreads = 512, kBwdThreads = 1024, kMaxLanes = 1024;
template <int NL, int MOST> struct NormShape {
  static constexpr int ROWS = NL < MOST ? MOST / NL : 1;     // rows at a time
  static constexpr int NT = ROWS * NL;
  static constexpr int WAVES = NL > kWave ? NL / kWave : 1;  // waves of a row
  // lanes that add the waves' parts: a power of two
  static constexpr int PARTS = WAVES > 8 ? 16 : WAVES > 4 ? 8 : WAVES > 2 ? 4 : WAVES;
};

// sum over the row's lanes inside a wave
template <int NL>
__device__ __forceinline__ float row_sum(float v) {
  return lanes_sum<(NL < kWave ? NL : kWave)>(v);
}

template <typename T, int NL, int VPL, bool RES>
__global__ __launch_bounds__((NormShape<NL, kFwdThreads>::NT)) void norm_fwd_kernel(
    const T* x, const T* residual, const float* __restrict__ gamma,
    const float* __restrict__ beta, unsigned n_rows, int d, float eps, T* sum_out,
    T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd) {
  using S = NormShape<NL, kFwdThreads>;
  constexpr int N = Vec<T>::N;
  __shared__ float s_red[2][S::NT / kWave][2];
  const int nvec = d / N;
  const int l = threadIdx.x % NL, sub = threadIdx.x / NL;
  const int wave = threadIdx.x / kWave, wave0 = wave - wave % S::WAVES;
  float g[VPL][N], b[VPL][N];
#pragma unroll
  for (int u = 0; u < VPL; ++u) {
    const int v = l + u * NL;
#pragma unroll
    for (int q = 0; q < N; ++q) g[u][q] = b[u][q] = 0.0f;
    if (v < nvec) {
      load_f32<N>(gamma + (size_t)v * N, g[u]);
      if (beta) load_f32<N>(beta + (size_t)v * N, b[u]);
    }
  }
  // columns of a row that its wave w holds
  auto cols_of = [&](int w) {
    if (NL <= kWave) return d;
    int n = 0;
#pragma unroll
    for (int u = 0; u < VPL; ++u) n += N * min(kWave, max(0, nvec - u * NL - w * kWave));
    return n;
  };
  const int cols = cols_of(wave % S::WAVES);
  const int w = threadIdx.x % S::PARTS;    // the wave whose part this lane adds
  const float cols_w = w < S::WAVES ? (float)cols_of(w) : 0.0f;
  Vec<T> xv[VPL], rv[VPL];
  auto load = [&](unsigned row) {
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      const int v = min(l + u * NL, nvec - 1);
      const size_t at = (size_t)min(row, n_rows - 1) * d + (size_t)v * N;
      xv[u].load(x + at);
      if (RES) rv[u].load(residual + at);
    }
  };
  const unsigned step = gridDim.x * S::ROWS;
  unsigned row = blockIdx.x * S::ROWS + sub;
  if (!RES) load(row);
  unsigned base = blockIdx.x * S::ROWS;   // < n_rows; rows and steps may pass int32
  for (int it = 0;; it ^= 1) {
    const bool more = n_rows - base > step;
    if (RES) load(row);
    float s[VPL][N];
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      const int v = l + u * NL;
#pragma unroll
      for (int q = 0; q < N; ++q) s[u][q] = 0.0f;
      if (row >= n_rows || v >= nvec) continue;
      xv[u].get(s[u]);
      if (RES) {
        float r[N];
        rv[u].get(r);
#pragma unroll
        for (int q = 0; q < N; ++q) s[u][q] += r[q];
        xv[u].put(s[u]);
        if (sum_out) xv[u].store(sum_out + (size_t)row * d + (size_t)v * N);
      }
#pragma unroll
      for (int q = 0; q < N; ++q) sum += s[u][q];
    }
    if (!RES && more) load(row + step);
    // the wave's own mean and centred squares; several waves' are merged by
    //   M2 = sum_w (M2_w + n_w (mu_w - mu)^2)
    float mu = cols ? row_sum<NL>(sum) / (float)cols : 0.0f;
    float sq = 0.0f;
#pragma unroll
    for (int u = 0; u < VPL; ++u)
      if (l + u * NL < nvec) {
#pragma unroll
        for (int q = 0; q < N; ++q) sq += (s[u][q] - mu) * (s[u][q] - mu);
      }
    sq = row_sum<NL>(sq);
    if constexpr (S::WAVES > 1) {
      if (threadIdx.x % kWave == 0) {
        s_red[it][wave][0] = mu;
        s_red[it][wave][1] = sq;
      }
      __syncthreads();
      const float* const part = s_red[it][wave0 + min(w, S::WAVES - 1)];
      const float mu_w = part[0], sq_w = w < S::WAVES ? part[1] : 0.0f;
      mu = lanes_sum<S::PARTS>(mu_w * cols_w) / (float)d;
      sq = lanes_sum<S::PARTS>(sq_w + cols_w * (mu_w - mu) * (mu_w - mu));
    }
    const float rs = 1.0f / sqrtf(sq / (float)d + eps);
    if (row < n_rows) {
#pragma unroll
      for (int u = 0; u < VPL; ++u) {
        const int v = l + u * NL;
        if (v >= nvec) continue;
        float o[N];
#pragma unroll
        for (int q = 0; q < N; ++q) o[q] = (s[u][q] - mu) * rs * g[u][q] + b[u][q];
        Vec<T> ov;
        ov.put(o);
        ov.store(y + (size_t)row * d + (size_t)v * N);
      }
      if (l == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = rs;
      }
    }
    if (!more) break;
    base += step;
    row += step;
  }
}

// dx of the rows a workgroup walks, and its rows' sums of dy xh and dy.
template <typename T, int NL, int VPL>
__global__ __launch_bounds__((NormShape<NL, kBwdThreads>::NT)) void norm_bwd_kernel(
    const T* dy, const T* __restrict__ sv, const float* __restrict__ gamma,
    const float* __restrict__ mean, const float* __restrict__ rstd, const T* dres,
    unsigned n_rows, int d, T* dx, float* __restrict__ sum_g, float* __restrict__ sum_b,
    int sum_stride) {
  using S = NormShape<NL, kBwdThreads>;
  constexpr int N = Vec<T>::N;
  // The next row, and gamma, in registers while these last: 16 columns a lane only with
  // up to 768 threads (3000 x 12288 bf16 61 us for 73; at 2000 x 14336, 896 threads, 78
  // for 58, and 2000 x 12288 float32, four vectors, 96 for 85).
  constexpr bool AHEAD = N * VPL <= 8 || (VPL == 2 && NL <= 768);
  __shared__ float s_red[2][S::NT / kWave][2];
  const int nvec = d / N;
  const int l = threadIdx.x % NL, sub = threadIdx.x / NL;
  const int wave = threadIdx.x / kWave, wave0 = wave - wave % S::WAVES;
  float held[AHEAD ? VPL : 1][N], wg[VPL][N], wb[VPL][N];
#pragma unroll
  for (int u = 0; u < VPL; ++u) {
    const int v = l + u * NL;
#pragma unroll
    for (int q = 0; q < N; ++q) wg[u][q] = wb[u][q] = 0.0f;
    if (AHEAD && v < nvec) load_f32<N>(gamma + (size_t)v * N, held[AHEAD ? u : 0]);
  }
  auto gamma_of = [&](int u, float g[N]) {   // of a vector inside the row
    if constexpr (AHEAD) {
#pragma unroll
      for (int q = 0; q < N; ++q) g[q] = held[u][q];
    } else {
      load_f32<N>(gamma + (size_t)(l + u * NL) * N, g);
    }
  };
  Vec<T> xv[VPL], yv[VPL], rv[VPL];
  float mu = 0.0f, rs = 0.0f;
  auto load = [&](unsigned row) {
    row = min(row, n_rows - 1);
    mu = mean[row];
    rs = rstd[row];
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      const size_t at = (size_t)row * d + (size_t)min(l + u * NL, nvec - 1) * N;
      xv[u].load(sv + at);
      yv[u].load(dy + at);
      if (dres) rv[u].load(dres + at);
    }
  };
  const unsigned step = gridDim.x * S::ROWS;
  unsigned row = blockIdx.x * S::ROWS + sub;
  if constexpr (AHEAD) load(row);
  unsigned base = blockIdx.x * S::ROWS;   // < n_rows; rows and steps may pass int32
  for (int it = 0;; it ^= 1) {
    const bool more = n_rows - base > step;
    if constexpr (!AHEAD) load(row);
    const bool on = row < n_rows;
    const float r1 = rs;
    float xh[VPL][N], dv[VPL][N];
    Vec<T> res[VPL];
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
#pragma unroll
      for (int q = 0; q < N; ++q) xh[u][q] = dv[u][q] = 0.0f;
      if (!on || l + u * NL >= nvec) continue;
      xv[u].get(xh[u]);
      yv[u].get(dv[u]);
      if (AHEAD && dres) res[u] = rv[u];
      float g[N];
      gamma_of(u, g);
#pragma unroll
      for (int q = 0; q < N; ++q) {
        xh[u][q] = (xh[u][q] - mu) * r1;
        a += g[q] * dv[u][q];
        b += g[q] * dv[u][q] * xh[u][q];
        wg[u][q] += dv[u][q] * xh[u][q];
        wb[u][q] += dv[u][q];
      }
    }
    if (AHEAD && more) load(row + step);
    a = row_sum<NL>(a);
    b = row_sum<NL>(b);
    if constexpr (S::WAVES > 1) {
      if (threadIdx.x % kWave == 0) {
        s_red[it][wave][0] = a;
        s_red[it][wave][1] = b;
      }
      __syncthreads();
      const int w = threadIdx.x % S::PARTS;
      const float* const part = s_red[it][wave0 + min(w, S::WAVES - 1)];
      a = lanes_sum<S::PARTS>(w < S::WAVES ? part[0] : 0.0f);
      b = lanes_sum<S::PARTS>(w < S::WAVES ? part[1] : 0.0f);
    }
    a /= (float)d;
    b /= (float)d;
#pragma unroll
    for (int u = 0; u < VPL; ++u) {
      const int v = l + u * NL;
      if (!on || v >= nvec) continue;
      float o[N], r[N], g[N];
      gamma_of(u, g);
#pragma unroll
      for (int q = 0; q < N; ++q) o[q] = r1 * (g[q] * dv[u][q] - a - xh[u][q] * b);
      if (dres) {
        (AHEAD ? res[u] : rv[u]).get(r);
#pragma unroll
        for (int q = 0; q < N; ++q) o[q] += r[q];
      }
      Vec<T> ov;
      ov.put(o);
      ov.store(dx + (size_t)row * d + (size_t)v * N);
    }
    if (!more) break;
    base += step;
    row += step;
  }
  if (!sum_g) return;
  // rows side by side in the workgroup: their sums added in order through LDS
  float* const outs[2] = {sum_g + (size_t)blockIdx.x * sum_stride,
                          sum_b ? sum_b + (size_t)blockIdx.x * sum_stride : nullptr};
  __shared__ float s_sum[S::ROWS > 1 ? S::ROWS * NL * N : 1];
#pragma unroll
  for (int u = 0; u < VPL; ++u)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float* const out = outs[which];
      if (!out) continue;  // (uniform)
      const float* const w = which ? wb[u] : wg[u];
      const int v = l + u * NL;
      if constexpr (S::ROWS == 1) {
        if (v < nvec) {
#pragma unroll
          for (int q = 0; q < N; q += 4)
            *reinterpret_cast<f32x4_t*>(out + (size_t)v * N + q) =
                f32x4_t{w[q], w[q + 1], w[q + 2], w[q + 3]};
        }
      } else {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < N; ++q) s_sum[(sub * NL + l) * N + q] = w[q];
        __syncthreads();
        for (int c = threadIdx.x; c < NL * N; c += S::NT) {
          float t = 0.0f;
#pragma unroll
          for (int i = 0; i < S::ROWS; ++i) t += s_sum[i * NL * N + c];
          const int col = u * NL * N + c;
          if (col < d) out[col] = t;
        }
      }
    }
}

// dgamma, dbeta: the workgroups' partial rows, 16 at a time side by side, the 16 sums
// in order.
constexpr int kRedCols = 64;   // columns per workgroup, four a thread
__global__ __launch_bounds__(256) void norm_bwd_reduce_kernel(const float* __restrict__ part,
                                                              int n_part, int d,
                                                              float* __restrict__ dgamma,
                                                              float* __restrict__ dbeta) {
  __shared__ __attribute__((aligned(16))) float s_sum[16][kRedCols];
  const int lane = threadIdx.x % 16, row = threadIdx.x / 16;
  const int c = blockIdx.x * kRedCols + lane * 4;   // of the 2 d columns (d % 8 == 0)
  f32x4_t t = {0.f, 0.f, 0.f, 0.f};
  if (c < 2 * d) {
    const float* const p = part + c;
    for (int i = row; i < n_part; i += 128) {   // eight loads in flight
      f32x4_t v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        v[u] = i + 16 * u < n_part
                   ? *reinterpret_cast<const f32x4_t*>(p + (size_t)(i + 16 * u) * 2 * d)
                   : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 8; ++u) t += v[u];
    }
  }
  *reinterpret_cast<f32x4_t*>(&s_sum[row][lane * 4]) = t;
  __syncthreads();
  const int col = blockIdx.x * kRedCols + threadIdx.x;
  if (threadIdx.x >= kRedCols || col >= 2 * d) return;
  float v = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += s_sum[i][threadIdx.x];
  if (col < d) dgamma[col] = v;
  else if (dbeta) dbeta[col - d] = v;
}

constexpr int kNormThreads = 256, kWideGroups = 1 << 16;
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

// Rows wider than the registers of a workgroup: one workgroup per row, read again
// for each of its passes (4096 x 20480 bf16 with a residual 220 us, 3.0 TB/s; the widest
// rows that stay in registers, 4096 x 16384, 94 us).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_wide_kernel(
    const T* x, const T* residual, const float* __restrict__ gamma,
    const float* __restrict__ beta, int n_rows, int d, float eps, T* sum_out,
    T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_red[kNormWaves];
  for (unsigned r = blockIdx.x; r < (unsigned)n_rows; r += gridDim.x) {
    const size_t row = (size_t)r * d;
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
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
}

// One workgroup per range of rows: dx of each, and the range's partial dgamma
// and dbeta rows, updated in place by the thread that owns the columns.  s and dy are read
// twice and the partial rows read and written for every row, by 256 threads: 4096 x 20480
// bf16 with dres 926 us (0.7 TB/s; 4096 x 16384, in registers, 115).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_wide_kernel(
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

// Workgroups of a call.  Forward: as many a CU as come nearest to these waves, with a
// residual and without one: with it 24 take 188 us for 181 at 32768 x 4096 bf16, 86 for 80
// at 30000 x 1000 float32, though 38 for 42 at 40000 x 640 bf16; without, 16 take 34 us
// for 28 at 24607 x 768 float32, 16 for 15 at 8192 x 2048 bf16, and 32 take 62 for 54 at
// 29392 x 2240; rounded down, 16-wave rows keep 16: 84 us for 66 at 12000 x 7168.  The
// numbers are the best over these sizes together; they know neither length nor width.
constexpr int kCus = 256, kFwdWaves = 19, kFwdWavesAlone = 24, kBwdGroups = 256;

// f(lanes per row, vectors per lane) for rows of d columns; false past 16384.
template <typename T, typename F>
bool norm_shape(int d, F f) {
  const int nvec = d / Vec<T>::N;
  const auto with = [&](auto nl, auto vpl) { return f(nl, vpl), true; };
  const std::integral_constant<int, 1> one{};
  if (nvec <= 8) return with(std::integral_constant<int, 8>{}, one);
  if (nvec <= 16) return with(std::integral_constant<int, 16>{}, one);
  if (nvec <= 32) return with(std::integral_constant<int, 32>{}, one);
  switch ((nvec + kWave - 1) / kWave) {
    case 1: return with(std::integral_constant<int, 64>{}, one);
    case 2: return with(std::integral_constant<int, 128>{}, one);
    case 3: return with(std::integral_constant<int, 192>{}, one);
    case 4: return with(std::integral_constant<int, 256>{}, one);
    case 5: return with(std::integral_constant<int, 320>{}, one);
    case 6: return with(std::integral_constant<int, 384>{}, one);
    case 7: return with(std::integral_constant<int, 448>{}, one);
    case 8: return with(std::integral_constant<int, 512>{}, one);
  }
  const auto wide = [&](auto vpl) {
    constexpr int TWO = 2 * kWave * decltype(vpl)::value;   // two waves' vectors
    switch ((nvec + TWO - 1) / TWO) {
      case 5: return with(std::integral_constant<int, 640>{}, vpl);
      case 6: return with(std::integral_constant<int, 768>{}, vpl);
      case 7: return with(std::integral_constant<int, 896>{}, vpl);
      default: return with(std::integral_constant<int, kMaxLanes>{}, vpl);
    }
  };
  if (nvec <= kMaxLanes) return wide(one);
  if (nvec <= 2 * kMaxLanes) return wide(std::integral_constant<int, 2>{});
  if (Vec<T>::N == 4 && nvec <= 4 * kMaxLanes)
    return wide(std::integral_constant<int, Vec<T>::N == 4 ? 4 : 2>{});
  return false;
}

inline int norm_parts(int T) { return T < kBwdGroups ? T : kBwdGroups; }

}  // namespace

size_t layer_norm_bwd_ws_bytes(int T, int d) {
  return (size_t)norm_parts(T) * 2 * d * sizeof(float);
}

namespace {

template <typename T>
hipError_t norm_fwd_t(const T* x, const T* residual, const float* gamma, const float* beta, int n,
                      int d, float eps, T* sum_out, T* y, float* mean, float* rstd,
                      hipStream_t s) {
  const bool fits = norm_shape<T>(d, [&](auto nl, auto vpl) {
    constexpr int NL = decltype(nl)::value, VPL = decltype(vpl)::value;
    using S = NormShape<NL, kFwdThreads>;
    const int need = (n - 1) / S::ROWS + 1;
    const auto run = [&](auto kernel, int waves) {
      constexpr int W = S::NT / kWave;
      const int per = (waves + W / 2) / W, most = kCus * (per > 1 ? per : 1);
      hipLaunchKernelGGL(kernel, dim3((unsigned)(need < most ? need : most)), dim3(S::NT), 0, s, x,
                         residual, gamma, beta, n, d, eps, sum_out, y, mean, rstd);
    };
    if (residual) run(norm_fwd_kernel<T, NL, VPL, true>, kFwdWaves);
    else run(norm_fwd_kernel<T, NL, VPL, false>, kFwdWavesAlone);
  });
  if (!fits)
    hipLaunchKernelGGL(norm_fwd_wide_kernel<T>, dim3((unsigned)(n < kWideGroups ? n : kWideGroups)),
                       dim3(kNormThreads), 0, s, x, residual, gamma, beta, n, d, eps, sum_out, y,
                       mean, rstd);
  return hipGetLastError();
}

}  // namespace

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

namespace {

template <typename T>
hipError_t norm_bwd_t(const T* dy, const T* sv, const float* gamma, const float* mean,
                      const float* rstd, const T* dres, int n, int d, T* dx, float* dgamma,
                      float* dbeta, float* part, hipStream_t s) {
  int grid = 0;
  bool done = false;
  const bool fits = n == 0 || norm_shape<T>(d, [&](auto nl, auto vpl) {
    constexpr int NL = decltype(nl)::value, VPL = decltype(vpl)::value;
    using S = NormShape<NL, kBwdThreads>;
    const int need = (n - 1) / S::ROWS + 1;
    grid = need < kBwdGroups ? need : kBwdGroups;
    // Up to four passes of its rows one workgroup takes them all: its sums are the
    // gradients, and there is no second launch (bf16, d 2048, 16 rows 9.0 us for 11.9;
    // d 4096, 8 rows 9.7 for 11.8, but with eight passes 16 for 12).
    done = grid == 1 || (dgamma && need <= 4);
    if (done) grid = 1;
    float* const sum_g = !dgamma ? nullptr : done ? dgamma : part;
    float* const sum_b = !dgamma ? nullptr : done ? dbeta : part + d;
    hipLaunchKernelGGL((norm_bwd_kernel<T, NL, VPL>), dim3((unsigned)grid), dim3(S::NT), 0, s, dy,
                       sv, gamma, mean, rstd, dres, n, d, dx, sum_g, sum_b, done ? 0 : 2 * d);
  });
  if (!fits) {
    const int per = (n - 1) / norm_parts(n) + 1;
    grid = (n - 1) / per + 1;
    hipLaunchKernelGGL(norm_bwd_wide_kernel<T>, dim3((unsigned)grid), dim3(kNormThreads), 0, s, dy,
                       sv, gamma, mean, rstd, dres, n, per, d, dx, dgamma ? part : nullptr);
  }
  if (dgamma && !done)
    hipLaunchKernelGGL(norm_bwd_reduce_kernel, dim3((unsigned)((2 * d + kRedCols - 1) / kRedCols)),
                       dim3(256), 0, s, part, grid, d, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace

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
