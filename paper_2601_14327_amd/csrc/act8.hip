// Activation checkpoints in 8 bits (moe_act8_save, moe_act8_load) and the SwiGLU
// backward at them (moe_swiglu_bwd_act8, moe_grouped_ffn_bwd_gather_act8).
// 32 consecutive columns of a row share a power-of-two scale, kept as its biased
// exponent b: with b = max(exponent of the block's largest magnitude - 6, 1),
//   q = clamp(round(v 2^(127 - b)), -127, 127),  the value it stands for q 2^(b - 127).
// Scaling by a power of two is exact, so rounding happens once, to the nearest of
// 127 steps (ties to even), and the decoded value is exact in bf16: |q| has 7
// bits.  From 2^-120 up the largest magnitude takes 64 to 127 steps, so the error is at
// most half a step, 1/128 of it (magnitudes above 127.5 steps, which no bf16 value is,
// lose up to one); below 2^-120 steps are 2^-126 and the error at most 2^-127.  A block
// with an infinity or a NaN has b = 255 and decodes to NaNs.
#include "common.hpp"
#include "internal.hpp"

namespace laep {
namespace {

// HBM-bound; 16 bytes of values a thread and no loop while the grid allows: 16 bf16
// columns a thread took 178 us and persistent grids of 1024 to 4096 workgroups 144 to
// 160 us against 132 (6.1 TB/s) for save and load of 65536 x 2048 bf16.  Stores stream:
// what they write is read much later, or by a product that reads it many times
// (ordinary ones: 141 us, and 122 against 111 in the SwiGLU backward at d_ff 1024).
constexpr int kActThreads = 256;
constexpr uint32_t kActNan = 255;

// A thread's 16 bytes of consecutive values: N of them, and their steps' bytes.  8
// float32 columns a thread, its two stores filling half of each 32 bytes, took 117 us
// instead of 90 for save and load of 24576 x 2048 and 56 instead of 41 for the SwiGLU
// backward of 12288 rows of d_ff 1024.
template <typename T> struct Run;
template <> struct Run<bf16_t> {
  static constexpr int N = 8;
  typedef u32x2_t Steps;
  u32x4_t r;
  template <bool STREAM> __device__ __forceinline__ void load(const bf16_t* p) {
    const u32x4_t* const at = reinterpret_cast<const u32x4_t*>(p);
    r = STREAM ? ld_stream(at) : *at;
  }
  __device__ __forceinline__ void get(float v[N]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = lo_bf16(r[i]);
      v[2 * i + 1] = hi_bf16(r[i]);
    }
  }
  __device__ static __forceinline__ void store(bf16_t* p, const float v[N]) {
    Elem<bf16_t>::store8_stream(p, v);
  }
};
template <> struct Run<float> {
  static constexpr int N = 4;
  typedef uint32_t Steps;
  f32x4_t r;
  template <bool STREAM> __device__ __forceinline__ void load(const float* p) {
    const f32x4_t* const at = reinterpret_cast<const f32x4_t*>(p);
    r = STREAM ? ld_stream(at) : *at;
  }
  __device__ __forceinline__ void get(float v[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = r[i];
  }
  __device__ static __forceinline__ void store(float* p, const float v[N]) {
    st_stream(reinterpret_cast<f32x4_t*>(p), f32x4_t{v[0], v[1], v[2], v[3]});
  }
};
__device__ __forceinline__ uint32_t word_of(u32x2_t q, int i) { return q[i]; }
__device__ __forceinline__ uint32_t word_of(uint32_t q, int) { return q; }

// largest magnitude of a block's neighbouring lanes (four or eight), as float bits: they
// order as unsigned integers, NaNs above infinity
template <int LANES>
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
  auto with = [&](int o) { v = v > (uint32_t)o ? v : (uint32_t)o; };
  with(__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
  with(__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
  if constexpr (LANES == 8) with(__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
  return v;
}

// biased exponent of the block's scale, from the bits of its largest magnitude
__device__ __forceinline__ uint32_t act8_exponent(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  return e == kActNan ? kActNan : (e > 7 ? e - 6 : 1);
}

__device__ __forceinline__ uint32_t act8_quant4(const float* v, float inv) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float q = fminf(fmaxf(rintf(v[i] * inv), -127.0f), 127.0f);
    w |= ((uint32_t)(int)q & 0xFFu) << (8 * i);
  }
  return w;
}

// the factor a block's steps decode with
__device__ __forceinline__ float act8_scale(uint32_t b) {
  return __uint_as_float(b == kActNan ? 0x7FC00000u : b << 23);
}

template <typename T>
__device__ __forceinline__ void act8_decode(typename Run<T>::Steps q, float scale, float* v) {
#pragma unroll
  for (int i = 0; i < Run<T>::N; ++i)
    v[i] = (float)(int8_t)(word_of(q, i >> 2) >> (8 * (i & 3))) * scale;
}

// One run per thread; 32 / N lanes share a block.  n_vec is a multiple of that, so a
// block's lanes are all in range or all out.
template <typename T>
__global__ __launch_bounds__(kActThreads) void act8_save_kernel(
    const T* __restrict__ act, long long n_vec, typename Run<T>::Steps* __restrict__ q,
    uint8_t* __restrict__ scale) {
  constexpr int N = Run<T>::N, LANES = 32 / N;
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < n_vec;
       i += (long long)gridDim.x * kActThreads) {
    Run<T> run;
    run.template load<false>(act + i * N);
    float v[N];
    run.get(v);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t a = __float_as_uint(v[e]) & 0x7FFFFFFFu;
      m = m > a ? m : a;
    }
    const uint32_t b = act8_exponent(block_max<LANES>(m));
    // a block that is not finite stores zeros: its exponent already says NaN
    const float inv = b == kActNan ? 0.0f : __uint_as_float((254u - b) << 23);
    typename Run<T>::Steps w{};
    if (b != kActNan) {
      if constexpr (N == 8) w = u32x2_t{act8_quant4(v, inv), act8_quant4(v + 4, inv)};
      else w = act8_quant4(v, inv);
    }
    __builtin_nontemporal_store(w, q + i);
    if (threadIdx.x % LANES == 0) scale[i / LANES] = (uint8_t)b;
  }
}

template <typename T>
__global__ __launch_bounds__(kActThreads) void act8_load_kernel(
    const typename Run<T>::Steps* __restrict__ q, const uint8_t* __restrict__ scale,
    long long n_vec, T* __restrict__ act) {
  constexpr int N = Run<T>::N, LANES = 32 / N;
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < n_vec;
       i += (long long)gridDim.x * kActThreads) {
    float v[N];
    act8_decode<T>(q[i], act8_scale(scale[i / LANES]), v);
    Run<T>::store(act + i * N, v);
  }
}

// SwiGLU backward, one run of one row per thread: with A_g and
// A_u decoded and s = sigmoid(A_g),
//   dA_g = dH A_u s (1 + A_g (1 - s)),  dA_u = dH silu(A_g),  H = silu(A_g) A_u.
// h may be dh (each thread reads its vector before it writes it).  STREAM: dh's loads
// stream, see the launch.
template <typename T, bool STREAM>
__global__ __launch_bounds__(kActThreads) void swiglu_bwd_act8_kernel(
    const typename Run<T>::Steps* __restrict__ q, const uint8_t* __restrict__ scale, const T* dh,
    long long R, int f, T* __restrict__ da, T* h) {
  constexpr int N = Run<T>::N, LANES = 32 / N;
  const int vpr = f / N;
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < R * vpr;
       i += (long long)gridDim.x * kActThreads) {
    const long long r = i / vpr;
    const int v = (int)(i % vpr);
    const long long g = r * 2 * vpr + v, u = g + vpr;
    float ag[N], au[N], d[N], og[N], ou[N], oh[N];
    act8_decode<T>(q[g], act8_scale(scale[g / LANES]), ag);
    act8_decode<T>(q[u], act8_scale(scale[u / LANES]), au);
    Run<T> run;
    run.template load<STREAM>(dh + i * N);
    run.get(d);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float sg = fast_sigmoid(ag[e]);
      const float sl = ag[e] * sg;
      og[e] = d[e] * au[e] * sg * (1.0f + ag[e] * (1.0f - sg));
      ou[e] = d[e] * sl;
      oh[e] = sl * au[e];
    }
    Run<T>::store(da + g * N, og);
    Run<T>::store(da + u * N, ou);
    Run<T>::store(h + i * N, oh);
  }
}

// (a grid dimension holds less than 2^32 threads; the kernels walk past the grid)
inline dim3 act_grid(long long n) {
  const long long g = (n + kActThreads - 1) / kActThreads;
  return dim3((unsigned)(g < 1 << 22 ? g : 1 << 22));
}

}  // namespace

namespace {

template <typename T>
hipError_t act8_save_t(const void* act, int64_t R, int C, void* q, uint8_t* scale, hipStream_t s) {
  const long long n = R * (long long)(C / Run<T>::N);
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(act8_save_kernel<T>, act_grid(n), dim3(kActThreads), 0, s,
                     static_cast<const T*>(act), n, static_cast<typename Run<T>::Steps*>(q),
                     scale);
  return hipGetLastError();
}

template <typename T>
hipError_t act8_load_t(const void* q, const uint8_t* scale, int64_t R, int C, void* act,
                       hipStream_t s) {
  const long long n = R * (long long)(C / Run<T>::N);
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(act8_load_kernel<T>, act_grid(n), dim3(kActThreads), 0, s,
                     static_cast<const typename Run<T>::Steps*>(q), scale, n,
                     static_cast<T*>(act));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_act8_save(const void* act, int dtype, int64_t R, int C, void* q, uint8_t* scale,
                            hipStream_t s) {
  return dtype == kDtypeBf16 ? act8_save_t<bf16_t>(act, R, C, q, scale, s)
                             : act8_save_t<float>(act, R, C, q, scale, s);
}

hipError_t launch_act8_load(const void* q, const uint8_t* scale, int dtype, int64_t R, int C,
                            void* act, hipStream_t s) {
  return dtype == kDtypeBf16 ? act8_load_t<bf16_t>(q, scale, R, C, act, s)
                             : act8_load_t<float>(q, scale, R, C, act, s);
}

namespace {

template <typename T, bool STREAM>
void swiglu_bwd_act8_t(const void* q, const uint8_t* scale, const void* dh, int64_t R, int f,
                       void* da, void* h, hipStream_t s) {
  hipLaunchKernelGGL((swiglu_bwd_act8_kernel<T, STREAM>), act_grid(R * (long long)(f / Run<T>::N)),
                     dim3(kActThreads), 0, s, static_cast<const typename Run<T>::Steps*>(q), scale,
                     static_cast<const T*>(dh), (long long)R, f, static_cast<T*>(da),
                     static_cast<T*>(h));
}

}  // namespace

hipError_t launch_swiglu_bwd_act8(const void* q, const uint8_t* scale, const void* dh, int dtype,
                                  int64_t R, int f, void* da, void* h, hipStream_t s) {
  if (R == 0) return hipSuccess;
  // dh, which the product before has just written, streams once the call's bytes pass
  // what the 256 MB last-level cache holds: 65536 rows of d_ff 1024 (675 MB) 117 us with
  // ordinary loads, 103 streaming; 12000 of 2048 (248 MB) 42.5 / 38.6; 3062 of 2048
  // (63 MB) 10.6 / 12.4.
  const int64_t elem = dtype == kDtypeBf16 ? 2 : 4;
  const bool stream = R * f * (2 + 4 * elem) > (int64_t)224 << 20;
  if (dtype == kDtypeBf16) {
    if (stream) swiglu_bwd_act8_t<bf16_t, true>(q, scale, dh, R, f, da, h, s);
    else swiglu_bwd_act8_t<bf16_t, false>(q, scale, dh, R, f, da, h, s);
  } else {
    if (stream) swiglu_bwd_act8_t<float, true>(q, scale, dh, R, f, da, h, s);
    else swiglu_bwd_act8_t<float, false>(q, scale, dh, R, f, da, h, s);
  }
  return hipGetLastError();
}

}  // namespace laep
