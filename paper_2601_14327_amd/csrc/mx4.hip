// Microscaled 4-bit matrices (moe_mx4_quantize, moe_mx4_dequantize).  Per 32 columns
//   b = max(exponent of the largest magnitude - 2, 0),  code = step nearest v 2^(127 - b):
// scaling by a power of two is exact, so rounding happens once.
// HBM-bound.  A workgroup takes rows of one group of 256 columns, whose eight scale bytes
// a row lie beside the next row's, so codes are written in whole 128-byte lines and
// scales in whole runs of rows.  64 x 2048 x 1024 in bf16 (340 MB): 56 us quantised (6.0
// TB/s), 48 us back (7.0, part of the codes still in the cache); 8 x 2048: 2.7 us each.
#include "common.hpp"
#include "internal.hpp"
#include "mx4.hpp"

namespace laep {
namespace {

constexpr int kMx4Threads = 256;
constexpr int kMx4Rows = 16;   // rows of a workgroup's tile: 128 bytes of scales

// A lane's 16 bytes of consecutive values: N of them, LANES to a block of 32.
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  typedef uint32_t Codes;
  __device__ static __forceinline__ void load(const bf16_t* p, float v[N]) {
    Elem<bf16_t>::load8_stream(p, v);
  }
  __device__ static __forceinline__ Codes encode(const float v[N], float scale) {
    return mx4_codes4(v[0], v[1], v[2], v[3], scale) |
           mx4_codes4(v[4], v[5], v[6], v[7], scale) << 16;
  }
  __device__ static __forceinline__ void store(bf16_t* p, Codes c, float scale) {
    st_stream(reinterpret_cast<u32x4_t*>(p), mx4_values8_bf16(c, scale));
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  typedef uint16_t Codes;
  __device__ static __forceinline__ void load(const float* p, float v[N]) {
    const f32x4_t r = ld_stream(reinterpret_cast<const f32x4_t*>(p));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i];
  }
  __device__ static __forceinline__ Codes encode(const float v[N], float scale) {
    return (Codes)mx4_codes4(v[0], v[1], v[2], v[3], scale);
  }
  __device__ static __forceinline__ void store(float* p, Codes c, float scale) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)c, scale, 0);
    const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)c, scale, 1);
    st_stream(reinterpret_cast<f32x4_t*>(p), f32x4_t{a[0], a[1], b[0], b[1]});
  }
};

// largest of a block's LANES neighbouring lanes (four or eight)
template <int LANES>
__device__ __forceinline__ uint32_t block_umax(uint32_t v) {
  v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
  if constexpr (LANES == 8)
    v = umax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  return v;
}

// Walks the tiles (kMx4Rows rows x 256 columns, groups innermost) of n matrices: fn(row
// over all matrices, column, column valid, index of the block's scale byte, first lane of
// the block).  A block's lanes are all valid or all not (C % 32 == 0).
template <typename T, typename Fn>
__device__ __forceinline__ void for_each_piece(int n, long long R, int C, Fn fn) {
  constexpr int N = Piece<T>::N, LANES = kMx4Block / N, PER_ROW = kMx4Group / N;
  const int G = (C + kMx4Group - 1) / kMx4Group;
  const long long row_tiles = (R + kMx4Rows - 1) / kMx4Rows;
  const int lr = threadIdx.x / PER_ROW, lc = threadIdx.x % PER_ROW;
  for (long long t = blockIdx.x; t < n * row_tiles * G; t += gridDim.x) {
    const int g = (int)(t % G);
    const long long m = t / G / row_tiles, r0 = t / G % row_tiles * kMx4Rows;
    const int c = g * kMx4Group + lc * N;
#pragma unroll
    for (int p = 0; p < kMx4Rows * PER_ROW / kMx4Threads; ++p) {
      const long long r = r0 + p * (kMx4Threads / PER_ROW) + lr;
      if (r < R)
        fn(m * R + r, c, c < C, ((m * G + g) * R + r) * 8 + lc / LANES, lc % LANES == 0);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kMx4Threads) void mx4_quantize_kernel(
    const T* __restrict__ src, int n, long long R, int C, uint8_t* __restrict__ codes,
    uint8_t* __restrict__ scale) {
  constexpr int N = Piece<T>::N;
  for_each_piece<T>(n, R, C, [&](long long row, int c, bool in, long long si, bool first) {
    float v[N] = {};
    if (in) Piece<T>::load(src + row * C + c, v);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m = umax(m, mag_bits(v[i]));
    const uint32_t b = mx4_exponent(block_umax<kMx4Block / N>(m));
    const typename Piece<T>::Codes w =
        b == kMx4Nan ? (typename Piece<T>::Codes)0 : Piece<T>::encode(v, mx4_scale(b));
    if (in) *reinterpret_cast<typename Piece<T>::Codes*>(codes + (row * C + c) / 2) = w;
    if (first) scale[si] = (uint8_t)b;   // (blocks past C: of zeros, so 0)
  });
}

template <typename T>
__global__ __launch_bounds__(kMx4Threads) void mx4_dequantize_kernel(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale, int n, long long R,
    int C, T* __restrict__ out) {
  for_each_piece<T>(n, R, C, [&](long long row, int c, bool in, long long si, bool) {
    if (in)
      Piece<T>::store(out + row * C + c,
                      *reinterpret_cast<const typename Piece<T>::Codes*>(codes + (row * C + c) / 2),
                      mx4_scale(scale[si]));
  });
}

// (a grid dimension holds less than 2^32 threads; the kernels walk past the grid)
inline dim3 mx4_grid(int n, int64_t R, int C) {
  const int64_t t = n * ((R + kMx4Rows - 1) / kMx4Rows) * mx4_groups(C);
  return dim3((unsigned)(t < 1 << 22 ? t : 1 << 22));
}

}  // namespace

hipError_t launch_mx4_quantize(const void* src, int dtype, int n, int64_t R, int C, uint8_t* codes,
                               uint8_t* scale, hipStream_t s) {
  if (n == 0 || R == 0) return hipSuccess;
  if (dtype == kDtypeBf16)
    hipLaunchKernelGGL(mx4_quantize_kernel<bf16_t>, mx4_grid(n, R, C), dim3(kMx4Threads), 0, s,
                       static_cast<const bf16_t*>(src), n, (long long)R, C, codes, scale);
  else
    hipLaunchKernelGGL(mx4_quantize_kernel<float>, mx4_grid(n, R, C), dim3(kMx4Threads), 0, s,
                       static_cast<const float*>(src), n, (long long)R, C, codes, scale);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scale, int dtype, int n,
                                 int64_t R, int C, void* out, hipStream_t s) {
  if (n == 0 || R == 0) return hipSuccess;
  if (dtype == kDtypeBf16)
    hipLaunchKernelGGL(mx4_dequantize_kernel<bf16_t>, mx4_grid(n, R, C), dim3(kMx4Threads), 0, s,
                       codes, scale, n, (long long)R, C, static_cast<bf16_t*>(out));
  else
    hipLaunchKernelGGL(mx4_dequantize_kernel<float>, mx4_grid(n, R, C), dim3(kMx4Threads), 0, s,
                       codes, scale, n, (long long)R, C, static_cast<float*>(out));
  return hipGetLastError();
}

}  // namespace laep
