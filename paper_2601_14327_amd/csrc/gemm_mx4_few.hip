// Grouped products at MX4 weights for few rows an expert (decoding): the products of
// gemm_mx4.hip in tiles of 32 rows x 64 weight rows.
//
// Every weight byte is used once, so the products are bound by streaming the weights.  A
// single token has one workgroup a CU and is bound by latencies one after the other: the
// offsets, row_src, and in each step first activations, whose loads the compiler puts ahead
// of the weights' copies and waits for, then the copies; nothing of the next step is in
// flight (gate/up, two steps a wave, 8.1 us for 18 MB; down, one step, 4.9 for 9 MB).
// The waves of a workgroup split K: wave w takes the 256-column steps w, w + 4, ..., 8 KB
// of codes each, which it copies into LDS of its own; nothing waits for another wave until
// the partial sums are added, in the waves' order.  Sixteen waves a CU, 128 KB in flight.
// (us for gate/up and down of 128 rows in 43 of 64 experts, d 2048, d_ff 1024, bf16 activations 19.0 + 10.9;
// eight waves a tile 22.5 + 11.5; two steps in flight a wave and eight waves a CU 19.7 +
// 13.6; a tile a wave, no sums to add, 23.8 + 13.1; weights streamed past the caches 20.4
// + 11.9.)
// Activations go from memory to registers; the FFN's X becomes MX4 there, so no launch
// and no buffer stand between it and the first product.  No tile list: every wave finds
// its tile from the expert offsets.  The bf16 gate/up kernel needs six registers more than
// the 128 that sixteen waves a CU leave, and keeps them in scratch.
#include "gemm_mx4.hpp"

namespace laep {
namespace {

constexpr int kFewBM = 32, kFewBN = 64, kFewSplit = 4;

// Activations: MX4 codes with scales, bf16, or bf16 that become MX4 here.
enum { FEW_CODES = 0, FEW_BF16 = 1, FEW_ROUND = 2 };

struct FewTile {
  int row0, rows, phys, nt;
};

// Tile `slot` of XCD `xcd`: tiles of kFewBM rows x n_tiles column blocks, experts in
// order, the row tiles of a column block innermost; each XCD takes a contiguous range.
// Four experts a lane, by every wave for itself.
__device__ __forceinline__ bool few_tile(int xcd, int slot, const int32_t* __restrict__ offsets,
                                         const int32_t* __restrict__ expert_map, int E,
                                         int n_tiles, int lane, FewTile& te) {
  int o[5], mt[4], phys[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 5; ++i) o[i] = offsets[min(4 * lane + i, E)];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = 4 * lane + i;
    phys[i] = e < E ? (expert_map ? expert_map[e] : e) : -1;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    mt[i] = phys[i] >= 0 ? (max(o[i + 1] - o[i], 0) + kFewBM - 1) / kFewBM : 0;
    sum += mt[i];
  }
  int inc = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int n = __shfl_up(inc, off, 64);
    if (lane >= off) inc += n;
  }
  const int total = __builtin_amdgcn_readlane(inc, 63) * n_tiles;
  const int per = (total + 7) >> 3;
  const int L = xcd * per + slot;
  if (slot >= per || L >= total) return false;  // (uniform)
  int at = L - (inc - sum) * n_tiles;
  const uint64_t has = __ballot(at >= 0 && at < sum * n_tiles);
  const int src = (int)__builtin_ctzll(has);
  // that lane's expert
  int row0 = 0, rows = 0, ph = 0, nt = 0;
  bool found = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int cnt = mt[i] * n_tiles;
    if (!found && at < cnt) {
      const int m = at % mt[i];
      nt = at / mt[i];
      row0 = o[i] + m * kFewBM;
      rows = min(kFewBM, o[i + 1] - o[i] - m * kFewBM);
      ph = phys[i];
      found = true;
    }
    at -= cnt;
  }
  te.row0 = __builtin_amdgcn_readlane(row0, src);
  te.rows = __builtin_amdgcn_readlane(rows, src);
  te.phys = __builtin_amdgcn_readlane(ph, src);
  te.nt = __builtin_amdgcn_readlane(nt, src);
  return true;
}

// largest magnitude of sixteen dwords of bf16, as bf16 bits
__device__ __forceinline__ uint32_t amax_bf16(const u32x4_t v[4]) {
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  u16x2_t m = {0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    m = __builtin_elementwise_max(
        m, __builtin_bit_cast(u16x2_t, v[i >> 2][i & 3] & 0x7FFF7FFFu));
  return m[0] > m[1] ? m[0] : m[1];
}

// 32 bf16 values in MX4: codes, and the block's exponent
__device__ __forceinline__ u32x4_t mx4_block_bf16(const u32x4_t v[4], uint32_t& b) {
  b = mx4_exponent(amax_bf16(v) << 16);
  const float scale = mx4_scale(b);
  u32x4_t c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t d0 = v[i][0], d1 = v[i][1], d2 = v[i][2], d3 = v[i][3];
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, d0), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, d1), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, d2), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2_t, d3), scale, 3);
    c[i] = b == kMx4Nan ? 0u : w;
  }
  return c;
}

template <int AKIND, int EPI>
__global__ __launch_bounds__(64 * kFewSplit, 4) void gemm_mx4_few_kernel(Mx4Params p) {
  constexpr bool CODES = AKIND == FEW_CODES, MX4 = AKIND != FEW_BF16;
  constexpr int STEP = kFewBN * 128, NDMA = STEP / 1024;
  constexpr int NA = CODES ? 4 : 16;             // 16-byte loads of a step's activations
  __shared__ __attribute__((aligned(1024))) char smem[kFewSplit * STEP];
  static_assert(kFewSplit * 32 * 64 * 4 <= sizeof(smem), "the partial sums");

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  FewTile te;
  const unsigned block = block_index();
  if (!few_tile(block & 7, block >> 3, p.offsets, p.expert_map, p.E, p.n_tiles_n, lane,
                te))
    return;

  const int G = (p.K + kMx4Group - 1) / kMx4Group;
  // the activations' row of this lane; rows past the tile's end: any valid row
  const int rr = min(lane & 31, te.rows - 1);
  const uint32_t row = p.row_src ? p.row_src[te.row0 + rr] / p.slots_k : rr;
  const long long row0 = p.row_src ? 0 : te.row0;
  const int a_row_bytes = CODES ? p.K / 2 : p.K * 2;
  const uint32_t a_off = row * (uint32_t)a_row_bytes + half * (CODES ? 64 : 256);
  const __amdgpu_buffer_rsrc_t a_rsrc = mx4_rsrc(static_cast<const char*>(p.A) + row0 * a_row_bytes);
  const __amdgpu_buffer_rsrc_t sa_rsrc = mx4_rsrc(CODES ? p.a_scale + row0 * 8 : p.b_scale);

  // weight row of row r of the tile: 32 gate rows and the same columns' up rows, or 64 in
  // order (a block past N does not occur: N % 64 == 0)
  const int col0 = EPI == MX4_GU ? te.nt * 32 : te.nt * 64;
  auto weight_row = [&](int r) {
    return EPI == MX4_GU && r >= 32 ? p.f + col0 + r - 32 : col0 + r;
  };
  // copy i of a step: rows 8i .. 8i + 7, this lane's chunk of one of them
  int l_row = lane >> 3, l_chunk = (lane & 7) ^ l_row;
  const __amdgpu_buffer_rsrc_t b_rsrc = mx4_rsrc(p.B + (long long)te.phys * p.N * (p.K / 2));
  const __amdgpu_buffer_rsrc_t sb_rsrc = mx4_rsrc(p.b_scale + (long long)te.phys * G * p.N * 8);
  const uint32_t sb_off = (col0 + (lane & 31)) * 8 + half * 4;
  char* const own = smem + wave * STEP;
  auto copy_step = [&](int g) {                  // (columns past K: zeros)
#pragma unroll
    for (int c = 0; c < NDMA; ++c) {
      const int lc = l_chunk ^ c;
      const uint32_t off = (uint32_t)weight_row(8 * c + l_row) * (uint32_t)(p.K / 2) + lc * 16;
      const uint32_t v[1] = {g * kMx4Group + lc * kMx4Block < p.K ? off : kDroppedCopy};
      dma_chunks<1, 64>(own + c * 1024, b_rsrc, v, g * 128, 0);
    }
  };
  struct Act {
    u32x4_t v[NA];
    uint32_t scale, w_scale[2];
  };
  auto load_act = [&](int g, Act& a) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      a.w_scale[j] = __builtin_amdgcn_raw_buffer_load_b32(
          sb_rsrc, sb_off, (g * p.N + j * (EPI == MX4_GU ? p.f : 32)) * 8, 0);
    if (CODES)
      a.scale = __builtin_amdgcn_raw_buffer_load_b32(sa_rsrc, row * 8 + half * 4,
                                                     (int)(g * p.a_rows * 8), 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {                // a block of 32 columns; past K: zeros
      const bool in = (g * 8 + half * 4 + s) * kMx4Block < p.K;
      const uint32_t at = in ? a_off + s * (CODES ? 16 : 64) : kDroppedCopy;
#pragma unroll
      for (int n = 0; n < NA / 4; ++n)
        a.v[s * (NA / 4) + n] = __builtin_bit_cast(
            u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, at + n * 16,
                                                           g * (CODES ? 128 : 512), 0));
    }
  };

  f32x16_t acc[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
  for (int g = wave; g < G; g += kFewSplit) {
    Act a;
    opaque(l_row, l_chunk);   // (offsets derived from them are not kept)
    copy_step(g);
    load_act(g, a);
    wait_vmcnt<0>();
    uint32_t sa = CODES ? a.scale : 0;
    u32x4_t fa[4];
    if constexpr (MX4) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if constexpr (CODES) {
          fa[s] = a.v[s];
        } else {
          uint32_t b;
          fa[s] = mx4_block_bf16(a.v + 4 * s, b);
          sa |= b << (8 * s);
        }
      }
    }
    int f_off = (lane & 31) * 128 + (((4 * half) ^ swz8(lane & 31)) << 4), f_zero = 0;
    opaque(f_off, f_zero);
    auto codes_of = [&](int j, int s) {
      // (32 rows on, the swizzle differs in its highest bit)
      return *reinterpret_cast<const u32x4_t*>(own + (f_off ^ (s << 4) ^ (j << 6)) + j * 4096);
    };
    if constexpr (MX4) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        acc[j] = mfma_mx4<0>(codes_of(j, 0), fa[0], a.w_scale[j], sa, acc[j]);
        acc[j] = mfma_mx4<1>(codes_of(j, 1), fa[1], a.w_scale[j], sa, acc[j]);
        acc[j] = mfma_mx4<2>(codes_of(j, 2), fa[2], a.w_scale[j], sa, acc[j]);
        acc[j] = mfma_mx4<3>(codes_of(j, 3), fa[3], a.w_scale[j], sa, acc[j]);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4_t c = codes_of(j, s);
          const float scale = mx4_scale(a.w_scale[j] >> (8 * s) & 255);
#pragma unroll
          for (int n = 0; n < 4; ++n)
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8_t, mx4_values8_bf16(c[n], scale)),
                __builtin_bit_cast(bf16x8_t, a.v[4 * s + n]), acc[j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);   // (one block's values at a time: 128 registers)
      }
    }
    wait_lgkm0();   // read, before the next step's copies
  }
  __syncthreads();
  // partial sums: [wave][fragment][quad][lane], 16 bytes each
  auto part = [&](int w, int j, int q, int l) {
    return reinterpret_cast<f32x4_t*>(smem + ((w * 2 + j) * 4 + q) * 1024 + l * 16);
  };
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *part(wave, j, q, lane) =
          f32x4_t{acc[j][4 * q], acc[j][4 * q + 1], acc[j][4 * q + 2], acc[j][4 * q + 3]};
  __syncthreads();
  // eight rows a wave, eight lanes a row: columns 4 c4 .. of each fragment
  const int r = wave * 8 + (lane >> 3), c4 = lane & 7;
  f32x4_t sum[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    sum[j] = *part(0, j, c4 >> 1, (c4 & 1) * 32 + r);
#pragma unroll
    for (int w = 1; w < kFewSplit; ++w) sum[j] += *part(w, j, c4 >> 1, (c4 & 1) * 32 + r);
  }
  const bool live = r < te.rows;
  const long long orow = (long long)te.row0 + r;
  auto packed = [](const f32x4_t& v) {
    return u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  };
  if constexpr (EPI == MX4_GU) {
    const int f = p.f, col = col0 + c4 * 4;
    f32x4_t h;
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = fast_silu(sum[0][i]) * sum[1][i];
    if constexpr (MX4) {
      uint32_t m = umax(umax(mag_bits(h[0]), mag_bits(h[1])), umax(mag_bits(h[2]), mag_bits(h[3])));
      m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true));
      m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, true));
      m = umax(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xF, 0xF, true));
      const uint32_t b = mx4_exponent(m);
      const uint32_t c = b == kMx4Nan ? 0 : mx4_codes4(h[0], h[1], h[2], h[3], mx4_scale(b));
      if (live) {
        *reinterpret_cast<uint16_t*>(static_cast<char*>(p.out) + orow * (f / 2) + col / 2) =
            (uint16_t)c;
        uint8_t* const sc = p.out_scale + ((long long)(col0 / kMx4Group) * p.out_rows + orow) * 8;
        const int blk = col0 / kMx4Block % 8;
        if (c4 == 0) sc[blk] = (uint8_t)b;
        // the blocks past f
        if (col0 + kMx4Block == f && c4 > blk) sc[c4] = 0;
      }
    } else if (live) {
      if (p.act) {
        *reinterpret_cast<u32x2_t*>(p.act + orow * 2 * f + col) = packed(sum[0]);
        *reinterpret_cast<u32x2_t*>(p.act + orow * 2 * f + f + col) = packed(sum[1]);
      }
      *reinterpret_cast<u32x2_t*>(static_cast<bf16_t*>(p.out) + orow * f + col) = packed(h);
    }
  } else if (live) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const long long at = orow * p.N + col0 + j * 32 + c4 * 4;
      if constexpr (EPI == MX4_STORE)
        *reinterpret_cast<u32x2_t*>(static_cast<bf16_t*>(p.out) + at) = packed(sum[j]);
      else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(p.out) + at) = sum[j];
    }
  }
}

template <int AKIND, int EPI>
hipError_t launch_few(const Mx4Params& p, int64_t R, hipStream_t s) {
  // sum of ceil(rows / kFewBM) over the experts with rows
  const int64_t tiles = (R / kFewBM + (R < p.E ? R : p.E)) * p.n_tiles_n;
  hipLaunchKernelGGL((gemm_mx4_few_kernel<AKIND, EPI>), tile_grid(tiles),
                     dim3(64 * kFewSplit), 0, s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_few(const Mx4Args& a, bool round, const int32_t* offsets,
                          const int32_t* expert_map, int E, int64_t R, hipStream_t s) {
  Mx4Params p = mx4_params(a);
  p.offsets = offsets;
  p.expert_map = expert_map;
  p.E = E;
  p.n_tiles_n = a.f ? a.f / 32 : a.N / 64;
  if (a.f) return round ? launch_few<FEW_ROUND, MX4_GU>(p, R, s) : launch_few<FEW_BF16, MX4_GU>(p, R, s);
  if (a.a_scale)
    return a.f32_out ? launch_few<FEW_CODES, MX4_STORE_F32>(p, R, s)
                     : launch_few<FEW_CODES, MX4_STORE>(p, R, s);
  return a.f32_out ? launch_few<FEW_BF16, MX4_STORE_F32>(p, R, s)
                   : launch_few<FEW_BF16, MX4_STORE>(p, R, s);
}

}  // namespace laep
