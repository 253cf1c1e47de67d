// Activation checkpoints in 8 bits (moe_act8_save, moe_act8_load) and the SwiGLU
// backward at them (moe_swiglu_bwd_act8, moe_grouped_ffn_bwd_gather_act8).
// 32 consecutive columns of a row share a power-of-two scale, kept as its biased
// exponent b: with b = max(exponent of the block's largest magnitude - 6, 1),
//   q = clamp(round(v 2^(127 - b)), -127, 127),  the value it stands for q 2^(b - 127).
// Scaling by a power of two is exact, so rounding happens once, to the nearest of
// 127 steps (ties to even), and the decoded value is exact in bf16: |q| has 7
// bits.  The largest magnitude takes 64 to 127 steps, so the error is at most half
// a step, 1/128 of it (magnitudes above 127.5 steps, which no bf16 value is, lose
// up to one).  A block with an infinity or a NaN has b = 255 and decodes to NaNs.
#include "common.hpp"
#include "internal.hpp"

namespace laep {
namespace {

// HBM-bound; one vector of 8 columns a thread and no loop while the grid allows: 16
// columns a thread took 178 us and persistent grids of 1024 to 4096 workgroups 144 to
// 160 us against 132 (6.1 TB/s) for save and load of 65536 x 2048 bf16.  Stores stream:
// what they write is read much later, or by a product that reads it many times
// (ordinary ones: 141 us, and 122 against 111 in the SwiGLU backward at d_ff 1024).
constexpr int kActThreads = 256;
constexpr uint32_t kActNan = 255;

// largest magnitude of four neighbouring lanes (one block of 32 columns), as
// float bits: they order as unsigned integers, NaNs above infinity
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const uint32_t a = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
  v = v > a ? v : a;
  const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);
  return v > b ? v : b;
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

__device__ __forceinline__ void act8_decode8(u32x2_t q, float scale, float v[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = (float)(int8_t)(q[i >> 2] >> (8 * (i & 3))) * scale;
}

// One vector of 8 columns per thread; four lanes share a block.  n_vec is a
// multiple of 4, so a block's lanes are all in range or all out.
template <typename T>
__global__ __launch_bounds__(kActThreads) void act8_save_kernel(const T* __restrict__ act,
                                                                long long n_vec,
                                                                u32x2_t* __restrict__ q,
                                                                uint8_t* __restrict__ scale) {
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < n_vec;
       i += (long long)gridDim.x * kActThreads) {
    float v[8];
    Elem<T>::load8(act + i * 8, v);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t a = __float_as_uint(v[e]) & 0x7FFFFFFFu;
      m = m > a ? m : a;
    }
    const uint32_t b = act8_exponent(quad_max(m));
    // a block that is not finite stores zeros: its exponent already says NaN
    const float inv = b == kActNan ? 0.0f : __uint_as_float((254u - b) << 23);
    u32x2_t w = {0u, 0u};
    if (b != kActNan) {
      w[0] = act8_quant4(v, inv);
      w[1] = act8_quant4(v + 4, inv);
    }
    __builtin_nontemporal_store(w, q + i);
    if ((threadIdx.x & 3) == 0) scale[i >> 2] = (uint8_t)b;
  }
}

template <typename T>
__global__ __launch_bounds__(kActThreads) void act8_load_kernel(const u32x2_t* __restrict__ q,
                                                                const uint8_t* __restrict__ scale,
                                                                long long n_vec,
                                                                T* __restrict__ act) {
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < n_vec;
       i += (long long)gridDim.x * kActThreads) {
    float v[8];
    act8_decode8(q[i], act8_scale(scale[i >> 2]), v);
    Elem<T>::store8_stream(act + i * 8, v);
  }
}

// SwiGLU backward, one vector of 8 columns of one row per thread: with A_g and
// A_u decoded and s = sigmoid(A_g),
//   dA_g = dH A_u s (1 + A_g (1 - s)),  dA_u = dH silu(A_g),  H = silu(A_g) A_u.
// h may be dh (each thread reads its vector before it writes it).  STREAM: dh's loads
// stream, see the launch.
template <typename T, bool STREAM>
__global__ __launch_bounds__(kActThreads) void swiglu_bwd_act8_kernel(
    const u32x2_t* __restrict__ q, const uint8_t* __restrict__ scale, const T* dh, long long R,
    int f, T* __restrict__ da, T* h) {
  const int vpr = f / 8;
  for (long long i = (long long)blockIdx.x * kActThreads + threadIdx.x; i < R * vpr;
       i += (long long)gridDim.x * kActThreads) {
    const long long r = i / vpr;
    const int v = (int)(i % vpr);
    const long long g = r * 2 * vpr + v, u = g + vpr;
    float ag[8], au[8], d[8], og[8], ou[8], oh[8];
    act8_decode8(q[g], act8_scale(scale[g >> 2]), ag);
    act8_decode8(q[u], act8_scale(scale[u >> 2]), au);
    if constexpr (STREAM) Elem<T>::load8_stream(dh + i * 8, d);
    else Elem<T>::load8(dh + i * 8, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float sg = fast_sigmoid(ag[e]);
      const float sl = ag[e] * sg;
      og[e] = d[e] * au[e] * sg * (1.0f + ag[e] * (1.0f - sg));
      ou[e] = d[e] * sl;
      oh[e] = sl * au[e];
    }
    Elem<T>::store8_stream(da + g * 8, og);
    Elem<T>::store8_stream(da + u * 8, ou);
    Elem<T>::store8_stream(h + i * 8, oh);
  }
}

// (a grid dimension holds less than 2^32 threads; the kernels walk past the grid)
inline dim3 act_grid(long long n) {
  const long long g = (n + kActThreads - 1) / kActThreads;
  return dim3((unsigned)(g < 1 << 22 ? g : 1 << 22));
}

}  // namespace

hipError_t launch_act8_save(const void* act, int dtype, int64_t R, int C, void* q, uint8_t* scale,
                            hipStream_t s) {
  const long long n = R * (long long)(C / 8);
  if (n == 0) return hipSuccess;
  if (dtype == kDtypeBf16)
    hipLaunchKernelGGL(act8_save_kernel<bf16_t>, act_grid(n), dim3(kActThreads), 0, s,
                       static_cast<const bf16_t*>(act), n, static_cast<u32x2_t*>(q), scale);
  else
    hipLaunchKernelGGL(act8_save_kernel<float>, act_grid(n), dim3(kActThreads), 0, s,
                       static_cast<const float*>(act), n, static_cast<u32x2_t*>(q), scale);
  return hipGetLastError();
}

hipError_t launch_act8_load(const void* q, const uint8_t* scale, int dtype, int64_t R, int C,
                            void* act, hipStream_t s) {
  const long long n = R * (long long)(C / 8);
  if (n == 0) return hipSuccess;
  if (dtype == kDtypeBf16)
    hipLaunchKernelGGL(act8_load_kernel<bf16_t>, act_grid(n), dim3(kActThreads), 0, s,
                       static_cast<const u32x2_t*>(q), scale, n, static_cast<bf16_t*>(act));
  else
    hipLaunchKernelGGL(act8_load_kernel<float>, act_grid(n), dim3(kActThreads), 0, s,
                       static_cast<const u32x2_t*>(q), scale, n, static_cast<float*>(act));
  return hipGetLastError();
}

namespace {

template <typename T, bool STREAM>
void swiglu_bwd_act8_t(const void* q, const uint8_t* scale, const void* dh, int64_t R, int f,
                       void* da, void* h, hipStream_t s) {
  hipLaunchKernelGGL((swiglu_bwd_act8_kernel<T, STREAM>), act_grid(R * (long long)(f / 8)),
                     dim3(kActThreads), 0, s, static_cast<const u32x2_t*>(q), scale,
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
