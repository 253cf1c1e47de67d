// Shared pieces of the grouped MX4 products.
#pragma once

#include <type_traits>

#include "gemm_common.hpp"
#include "mx4.hpp"

namespace laep {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// Activations of a product: MX4 codes, or bf16.
enum { ACT_MX4 = 0, ACT_BF16 = 1 };
// Epilogues: SwiGLU to H (MX4 or bf16, as the activations), the product in bf16 or float32.
enum { MX4_GU = 0, MX4_STORE = 1, MX4_STORE_F32 = 2 };

constexpr uint32_t kDroppedCopy = 0x80000000u;  // past every descriptor: the copy writes zeros
constexpr int kMx4Extent = 0x7FFFFFFF;          // (host-checked: offsets lie below 2^31)

struct Mx4Params {
  const void* A;              // codes [rows, K / 2] or bf16 [rows, K]
  const uint8_t* a_scale;     // MX4: [G, a_rows, 8]
  int64_t a_rows;             // rows of the whole A
  const uint8_t* B;           // codes [slots, N, K / 2]
  const uint8_t* b_scale;     // [slots, G, N, 8]
  int N, K;
  int f;                      // SwiGLU: N = 2 f
  const int32_t* offsets;
  const int32_t* expert_map;
  int E;
  int n_tiles_n;
  void* out;                  // H (codes [R, f / 2] or bf16 [R, f]) or the product [R, N]
  uint8_t* out_scale;         // H's scales [ceil(f / 256), R, 8]
  int64_t out_rows;           // R
  bf16_t* act;                // SwiGLU: pre-activations [R, 2f] or NULL
  const int32_t* row_src;     // gathered A rows, or NULL
  int slots_k;
  const TileEntry* table;     // persistent products: the list of their tiles
  const int* n_entries;
};

inline Mx4Params mx4_params(const Mx4Args& a) {
  Mx4Params p = {};
  p.A = a.A;
  p.a_scale = a.a_scale;
  p.a_rows = a.a_rows;
  p.B = a.B;
  p.b_scale = a.b_scale;
  p.N = a.N;
  p.K = a.K;
  p.f = a.f;
  p.out = a.out;
  p.out_scale = a.out_scale;
  p.out_rows = a.out_rows;
  p.act = static_cast<bf16_t*>(a.act);
  p.row_src = a.row_src;
  p.slots_k = a.slots_k;
  return p;
}

// One 32 x 32 x 64 step of MX4 operands; byte S of a scale dword is the lane's block's.
template <int S>
__device__ __forceinline__ f32x16_t mfma_mx4(const u32x4_t& a, const u32x4_t& b, uint32_t sa,
                                             uint32_t sb, const f32x16_t& c) {
  const i32x8_t va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8_t vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(va, vb, c, 4, 4, S, (int)sa, S, (int)sb);
}

// copies of a step J (mod 4) of the bf16 products: its activations, and in the first two
// of four half of the next 256 columns of weights each, with their scales in the first
template <int NA, int NB>
constexpr int copies_of(int j) {
  return NA + (j % 4 == 0 ? NB / 2 + 1 : j % 4 == 1 ? NB / 2 : 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx4_rsrc(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, kMx4Extent, kBufferFlags);
}

// Global -> LDS copy of one dword a lane (a row's scales of four blocks): lane i at + 4 i.
__device__ __forceinline__ void dma_scales(char* dst, __amdgpu_buffer_rsrc_t rsrc, uint32_t voff,
                                           int soff, int wave) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void_t*)(dst + wave * 256), 4, voff, soff, 0,
                                           0);
}

// values the compiler knows nothing about from here on
template <typename T>
__device__ __forceinline__ void opaque(T& a, T& b) {
  asm volatile("" : "+v"(a), "+v"(b));
}

// H of one row's 32 columns in MX4: half the columns are in lane l, half in lane l ^ 32
// (h[4q + i] is column 8q + 4 (l / 32) + i).  Returns the block's exponent, and in w the
// eight bytes of codes that this lane stores (bytes 8 (l / 32) .. of the block's 16).
__device__ __forceinline__ uint32_t mx4_row_block(const float h[16], u32x2_t& w) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = umax(m, mag_bits(h[i]));
  const auto both = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  const uint32_t b = mx4_exponent(umax(both[0], both[1]));
  const float scale = mx4_scale(b);
  uint32_t c[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    c[q] = b == kMx4Nan ? 0u : mx4_codes4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3], scale);
  // the lower lanes take quads 0 and 1 of both halves, the upper ones 2 and 3
  const auto x = __builtin_amdgcn_permlane32_swap(c[0] | c[1] << 16, c[2] | c[3] << 16, false, false);
  w[0] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
  w[1] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
  return b;
}

// Stores a lane's part of a row's block of H; the lower half's lanes write its scale, and
// those of the last block the zeros of the blocks past f.
__device__ __forceinline__ void store_h_block(const Mx4Params& p, long long row, int fcol, int f,
                                              int half, const u32x2_t& w, uint32_t b) {
  *reinterpret_cast<u32x2_t*>(static_cast<char*>(p.out) + row * (f / 2) + fcol / 2 + half * 8) = w;
  if (half) return;
  uint8_t* const s = p.out_scale + ((fcol / kMx4Group) * p.out_rows + row) * 8;
  s[fcol / kMx4Block % 8] = (uint8_t)b;
  if (fcol + kMx4Block == f)
    for (int i = f / kMx4Block; i % 8; ++i) s[i % 8] = 0;
}

}  // namespace
}  // namespace laep
