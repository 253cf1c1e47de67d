// Grouped products at MX4 weights (moe_mx4_grouped_product, moe_grouped_ffn_fwd_mx4):
//   gate/up   A = X_e [M_e, d] x W_gu^T  -> SwiGLU epilogue (H in MX4 or bf16)
//   down      H_e [M_e, f] x W_d^T -> Y;  or the product alone, in bf16 or float32
// with X and H in MX4 (v_mfma_scale_f32_32x32x64_f8f6f4, four times the bf16 rate) or in
// bf16 (the weights' codes become bf16 in registers, exactly, by one instruction a pair,
// for v_mfma_f32_32x32x16_bf16).
//
// A k-step is 128 bytes of an activation row: 256 columns in MX4, 64 in bf16.  In MX4
// the lane halves take columns 0..127 and 128..255 of the step, sub-step s block s of
// the half, so one dword of a row's scales serves the lane's four sub-steps.  In bf16 a
// step's two blocks of 32 columns go to the two halves, sub-step s columns 8 s of each,
// and the weights' k-step of 256 columns serves four of the activations'.
#include <type_traits>

#include "gemm_mx4.hpp"

namespace laep {
namespace {

constexpr int kMx4GemmThreads = 256;
static_assert(kMx4GemmThreads == kTableThreads, "one thread per expert in find_tile");

// ---------------------------------------------------------------------------
// Tiles of BM x 128 in four waves (2 x 2, each BM/2 x 64): a ring of NST k-steps of
// activations (MX4: with the weights and both scales) and, for bf16, two 256-column steps
// of weights, in at most 80 KB, so that two workgroups share a CU (rings of two steps at 64
// rows: 52 KB, three).
// ---------------------------------------------------------------------------
template <int BM, int NST, int ACT, int EPI>
__global__ __launch_bounds__(kMx4GemmThreads) void gemm_mx4_kernel(Mx4Params p) {
  constexpr int BN = 128, NT = kMx4GemmThreads;
  constexpr int WTM = BM / 2, TM = WTM / 32, TN = 2;
  constexpr int ABYTES = BM * 128, BBYTES = BN * 128;
  constexpr int SBYTES = 1024;                       // an operand's scales of 256 columns
  constexpr bool MX4 = ACT == ACT_MX4;
  constexpr int NA = BM * 8 / NT, NB = BN * 8 / NT;
  static_assert(BM == 64 || BM == 128, "two rows of waves; an operand's scales fit 1 KB");
  constexpr int STAGE = MX4 ? ABYTES + BBYTES + 2 * SBYTES : ABYTES;
  constexpr int BSTAGE = BBYTES + SBYTES;            // bf16: the weights' own ring of two
  constexpr int SMEM = NST * STAGE + (MX4 ? 0 : 2 * BSTAGE);
  constexpr int PITCH = BN * 2 + 16;                 // bytes per staged output row
  static_assert(BM * PITCH <= SMEM && SMEM <= 80 * 1024, "staging fits, two workgroups a CU");
  static_assert(NST >= 2 && NST <= 4, "bf16: weights land three steps after their issue");
  __shared__ __attribute__((aligned(1024))) char smem[SMEM];

  const int tid = threadIdx.x;
  const int wave = tid >> 6, lane = tid & 63, half = lane >> 5;
  const int wave_s = __builtin_amdgcn_readfirstlane(wave);
  FoundTile te;
  if (!find_tile(block_index(), p.offsets, p.expert_map, p.E, BM, p.n_tiles_n, smem, te)) return;
  const int nt = te.nt;
  const int wm = wave / 2, wn = wave % 2;

  // weight row of B-tile row r: SwiGLU tiles hold 32 gate rows and the same columns' up
  // rows per 64, so a wave owns both
  auto weight_row = [&](int r) {
    if (EPI == MX4_GU) {
      const int w = r & 63, fcol = nt * (BN / 2) + (r >> 6) * 32 + (w & 31);
      return w < 32 ? fcol : p.f + fcol;
    }
    const int row = nt * BN + r;
    return row < p.N ? row : p.N - 1;
  };
  auto act_row = [&](int r) {  // rows past the tile's end: any valid row
    const int rr = r < te.rows ? r : te.rows - 1;
    return p.row_src ? p.row_src[te.row0 + rr] / p.slots_k : rr;
  };
  const int a_row_bytes = MX4 ? p.K / 2 : p.K * 2;
  uint32_t a_voff[NA], b_voff[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const int q = i * NT + tid, r = q >> 3, lc = (q & 7) ^ swz8(r);
    a_voff[i] = (uint32_t)(act_row(r) * (long long)a_row_bytes + lc * 16);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int q = i * NT + tid, r = q >> 3, lc = (q & 7) ^ swz8(r);
    b_voff[i] = (uint32_t)(weight_row(r) * (long long)(p.K / 2) + lc * 16);
  }
  const uint32_t sa_voff =
      MX4 ? (uint32_t)(act_row(min(tid >> 1, BM - 1)) * 8 + (tid & 1) * 4) : 0;
  const uint32_t sb_voff = (uint32_t)(weight_row(tid >> 1) * 8 + (tid & 1) * 4);
  const int G = (p.K + kMx4Group - 1) / kMx4Group;
  const long long row0 = p.row_src ? 0 : te.row0;
  const __amdgpu_buffer_rsrc_t a_rsrc = mx4_rsrc(static_cast<const char*>(p.A) + row0 * a_row_bytes);
  const __amdgpu_buffer_rsrc_t sa_rsrc = mx4_rsrc(MX4 ? p.a_scale + row0 * 8 : p.b_scale);
  const __amdgpu_buffer_rsrc_t b_rsrc = mx4_rsrc(p.B + (long long)te.phys * p.N * (p.K / 2));
  const __amdgpu_buffer_rsrc_t sb_rsrc = mx4_rsrc(p.b_scale + (long long)te.phys * G * p.N * 8);

  const int steps = MX4 ? G : p.K / 64;
  auto a_stage = [&](int t) { return smem + (t % NST) * STAGE; };
  auto b_stage = [&](int g) { return smem + NST * STAGE + (g & 1) * BSTAGE; };  // bf16
  // copies past the end are dropped (zeros that nobody reads), so that every step issues
  // the same number; in MX4 so are the columns of the last 256 that lie past K
  auto codes_at = [&](uint32_t voff, int i, int g) {
    const int q = i * NT + tid, lc = (q & 7) ^ swz8(q >> 3);
    return g * kMx4Group + lc * kMx4Block < p.K ? voff : kDroppedCopy;
  };
  auto issue_b = [&](char* dst, int i, int g) {
    const uint32_t v[1] = {codes_at(b_voff[i], i, g)};
    dma_chunks<1, NT>(dst + i * NT * 16, b_rsrc, v, g * 128, wave_s);
  };
  auto issue_sb = [&](char* dst, int g) {
    dma_scales(dst, sb_rsrc, g < G ? sb_voff : kDroppedCopy, min(g, G - 1) * p.N * 8, wave_s);
  };
  auto issue_a = [&](int t) {
    char* const st = a_stage(t);
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const uint32_t v[1] = {MX4 ? codes_at(a_voff[i], i, t) : t < steps ? a_voff[i] : kDroppedCopy};
      dma_chunks<1, NT>(st + i * NT * 16, a_rsrc, v, t * 128, wave_s);
    }
  };
  auto issue_mx4 = [&](int t) {
    char* const st = a_stage(t);
#pragma unroll
    for (int i = 0; i < NB; ++i) issue_b(st + ABYTES, i, t);
    issue_a(t);
    dma_scales(st + ABYTES + BBYTES, sa_rsrc, t < G ? sa_voff : kDroppedCopy,
               (int)(min(t, G - 1) * p.a_rows * 8), wave_s);
    issue_sb(st + ABYTES + BBYTES + SBYTES, t);
  };

  // fragment byte offsets: of sub-step 0 (MX4 both operands, bf16 the activations:
  // sub-step s ^ 16 s); the bf16 product's weights: step j of 256 columns ^ 32 j
  int a_off[TM], b_off[TN], a_row[TM], b_row[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = a_row[i] = wm * WTM + i * 32 + (lane & 31);
    a_off[i] = r * 128 + (((4 * half) ^ swz8(r)) << 4);
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int r = b_row[j] = wn * 64 + j * 32 + (lane & 31);
    b_off[j] = r * 128 + (((MX4 ? 4 * half : half) ^ swz8(r)) << 4);
  }
  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  if constexpr (MX4) {
    constexpr int NC = NA + NB + 2;
#pragma unroll
    for (int t = 0; t < NST - 1; ++t) issue_mx4(t);
    for (int t = 0; t < steps; ++t) {
      // step t has landed (the steps issued after it may be in flight); past the barrier
      // that holds for every thread, and step t - 1's stage is read and free
      wait_vmcnt<(NST - 2) * NC>();
      __builtin_amdgcn_s_barrier();
      issue_mx4(t + NST - 1);
      const char* const st = a_stage(t);
      const char* const sc = st + ABYTES + BBYTES + half * 4;
      u32x4_t fa[4][TM], fb[4][TN];
      uint32_t sa[TM], sb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j)
        sb[j] = *reinterpret_cast<const uint32_t*>(sc + SBYTES + b_row[j] * 8);
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(sc + a_row[i] * 8);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
          fb[s][j] = *reinterpret_cast<const u32x4_t*>(st + ABYTES + (b_off[j] ^ (s << 4)));
#pragma unroll
        for (int i = 0; i < TM; ++i)
          fa[s][i] = *reinterpret_cast<const u32x4_t*>(st + (a_off[i] ^ (s << 4)));
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          acc[i][j] = mfma_mx4<0>(fb[0][j], fa[0][i], sb[j], sa[i], acc[i][j]);
          acc[i][j] = mfma_mx4<1>(fb[1][j], fa[1][i], sb[j], sa[i], acc[i][j]);
          acc[i][j] = mfma_mx4<2>(fb[2][j], fa[2][i], sb[j], sa[i], acc[i][j]);
          acc[i][j] = mfma_mx4<3>(fb[3][j], fa[3][i], sb[j], sa[i], acc[i][j]);
        }
      wait_lgkm0();  // this step's reads are in registers before the next barrier frees it
    }
  } else {
    // The weights of 256 columns are issued in the first two of the four steps before
    // theirs (half each, with the scales in the first), so that the waits below, which
    // let NST - 2 steps' copies be in flight, find them landed.
#pragma unroll
    for (int i = 0; i < NB; ++i) issue_b(b_stage(0), i, 0);
    issue_sb(b_stage(0) + BBYTES, 0);
#pragma unroll
    for (int t = 0; t < NST - 1; ++t) issue_a(t);
    for (int g = 0; g < G; ++g) {
      const char* const bs = b_stage(g);
      auto step = [&](auto j_tag) {
        constexpr int J = decltype(j_tag)::value;
        const int t = 4 * g + J;
        if (t >= steps) return;
        // copies issued after step t's activations: those of the NST - 2 steps before
        // this one (before the loop only activations: fewer, so the first group waits
        // for those alone)
        constexpr int AHEAD = (NST > 2 ? copies_of<NA, NB>(J + 3) : 0) +
                              (NST > 3 ? copies_of<NA, NB>(J + 2) : 0);
        if (g == 0) wait_vmcnt<(NST - 2) * NA>();
        else wait_vmcnt<AHEAD>();
        __builtin_amdgcn_s_barrier();
        if constexpr (J == 0) issue_sb(b_stage(g + 1) + BBYTES, g + 1);
        if constexpr (J < 2) {
#pragma unroll
          for (int i = J * NB / 2; i < (J + 1) * NB / 2; ++i) issue_b(b_stage(g + 1), i, g + 1);
        }
        issue_a(t + NST - 1);
        const char* const st = a_stage(t);
        u32x4_t fa[4][TM], fb[TN];
        uint32_t sb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          sb[j] = *reinterpret_cast<const uint32_t*>(bs + BBYTES + b_row[j] * 8 + (J >> 1) * 4);
          fb[j] = *reinterpret_cast<const u32x4_t*>(bs + (b_off[j] ^ (J << 5)));
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int i = 0; i < TM; ++i)
            fa[s][i] = *reinterpret_cast<const u32x4_t*>(st + (a_off[i] ^ (s << 4)));
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const float scale = mx4_scale((sb[j] >> (16 * (J & 1) + 8 * half)) & 255);
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const bf16x8_t wv = __builtin_bit_cast(bf16x8_t, mx4_values8_bf16(fb[j][s], scale));
#pragma unroll
            for (int i = 0; i < TM; ++i)
              acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  wv, __builtin_bit_cast(bf16x8_t, fa[s][i]), acc[i][j], 0, 0, 0);
          }
        }
        wait_lgkm0();
      };
      step(std::integral_constant<int, 0>{});
      step(std::integral_constant<int, 1>{});
      step(std::integral_constant<int, 2>{});
      step(std::integral_constant<int, 3>{});
    }
  }
  wait_vmcnt<0>();               // dropped copies write zeros into the ring, too
  __builtin_amdgcn_s_barrier();  // every wave's reads are done: the ring is free for staging

  // ---- epilogue: the lane owns row lane % 32 of each block, columns 8q + 4 half + 0..3
  // of each fragment
  const int lrow = lane & 31;
  auto stage = [&](int row, int col, float a, float b, float c, float d) {
    u32x2_t w = {pack_bf16x2(a, b), pack_bf16x2(c, d)};
    *reinterpret_cast<u32x2_t*>(smem + row * PITCH + col * 2) = w;
  };
  auto sync = [&]() {
    wait_lgkm0();
    __builtin_amdgcn_s_barrier();
  };
  // staged columns [scol0, scol0 + 8 * CPR) -> dst + (te.row0 + row) * ld
  auto flush = [&](auto cpr_tag, bf16_t* dst, long long ld, int ncols, int scol0) {
    constexpr int CPR = decltype(cpr_tag)::value;
#pragma unroll
    for (int c = tid; c < BM * CPR; c += NT) {
      const int r = c / CPR, cc = c % CPR;
      if (r < te.rows && cc * 8 < ncols)
        *reinterpret_cast<u32x4_t*>(dst + ((long long)te.row0 + r) * ld + cc * 8) =
            *reinterpret_cast<const u32x4_t*>(smem + r * PITCH + (scol0 + cc * 8) * 2);
    }
  };
  if constexpr (EPI == MX4_GU && MX4) {
    const int fcol = nt * (BN / 2) + wn * 32, f = p.f;  // f % 64 == 0: whole blocks
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float h[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) h[r] = fast_silu(acc[i][0][r]) * acc[i][1][r];
      u32x2_t w;
      const uint32_t b = mx4_row_block(h, w);
      const int r = wm * WTM + i * 32 + lrow;
      if (r < te.rows)
        store_h_block(p, (long long)te.row0 + r, fcol, f, half, w, b);
    }
  } else if constexpr (EPI == MX4_GU) {
    const int f = p.f, fbase = nt * (BN / 2);
    using Half = std::integral_constant<int, BN / 16>;
    if (p.act) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            stage(wm * WTM + i * 32 + lrow, j * (BN / 2) + wn * 32 + q * 8 + half * 4,
                  acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                  acc[i][j][4 * q + 3]);
      sync();
      flush(Half{}, p.act + fbase, 2LL * f, BN / 2, 0);
      flush(Half{}, p.act + f + fbase, 2LL * f, BN / 2, BN / 2);
      sync();
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float h[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) h[u] = fast_silu(acc[i][0][4 * q + u]) * acc[i][1][4 * q + u];
        stage(wm * WTM + i * 32 + lrow, wn * 32 + q * 8 + half * 4, h[0], h[1], h[2], h[3]);
      }
    sync();
    flush(Half{}, static_cast<bf16_t*>(p.out) + fbase, f, BN / 2, 0);
  } else if constexpr (EPI == MX4_STORE) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          stage(wm * WTM + i * 32 + lrow, wn * 64 + j * 32 + q * 8 + half * 4, acc[i][j][4 * q],
                acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    sync();
    flush(std::integral_constant<int, BN / 8>{}, static_cast<bf16_t*>(p.out) + nt * BN, p.N,
          min(BN, p.N - nt * BN), 0);
  } else {
    float* const out = static_cast<float*>(p.out);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int r = wm * WTM + i * 32 + lrow;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = nt * BN + wn * 64 + j * 32 + q * 8 + half * 4;
          if (r < te.rows && col < p.N)
            *reinterpret_cast<f32x4_t*>(out + ((long long)te.row0 + r) * p.N + col) =
                f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                        acc[i][j][4 * q + 3]};
        }
    }
  }
}

// sum of ceil(rows / bm) over the experts with rows, at most
inline int64_t most_tiles(const Mx4Params& p, int bm, int64_t R) {
  return (R / bm + (R < p.E ? R : p.E)) * p.n_tiles_n;
}

template <int BM, int NST, int ACT, int EPI>
hipError_t launch_tiles(const Mx4Params& p, int64_t R, hipStream_t s) {
  const int64_t tiles = most_tiles(p, BM, R);
  if (tiles <= 0) return hipSuccess;
  hipLaunchKernelGGL((gemm_mx4_kernel<BM, NST, ACT, EPI>), tile_grid(tiles),
                     dim3(kMx4GemmThreads), 0, s, p);
  return hipGetLastError();
}

template <int ACT, int EPI>
hipError_t launch_middle(Mx4Params p, int bm, int64_t R, hipStream_t s) {
  p.n_tiles_n = EPI == MX4_GU ? p.f / 64 : ceil_div(p.N, 128);
  if (bm == 128) return launch_tiles<128, 2, ACT, EPI>(p, R, s);
  // More tiles than two a CU: rings of two steps, so that three fit (us for 3062 rows of 64
  // experts, 1088 x 1216, bf16 23.9 -> 19.9, 1500 rows 22.6 -> 18.7, MX4 16.0 -> 13.9); else
  // copies further ahead (1024 rows of one expert, 2048 x 2048, bf16 16.3, by two steps 18.4;
  // 2048 rows of 32, 1024 x 1024, MX4 9.2, by two 10.0).
  if (most_tiles(p, 64, R) > 512) return launch_tiles<64, 2, ACT, EPI>(p, R, s);
  return launch_tiles<64, ACT == ACT_MX4 ? 3 : 4, ACT, EPI>(p, R, s);
}

// The tiles of a product over E experts: 32 x 64 for few rows an expert (FEW), 64 or 128 x
// 128, or the persistent 128 or 256 x 256 (BIG).
enum Tiles { FEW, MID64, MID128, BIG128, BIG256 };
inline bool is_big(Tiles t) { return t >= BIG128; }
inline int rows_of(Tiles t) { return t == BIG256 ? 256 : t == FEW ? 32 : t == MID64 ? 64 : 128; }
inline int cols_of(Tiles t) { return is_big(t) ? 256 : t == FEW ? 64 : 128; }

// Which: the host knows neither the loads nor how many experts have rows, so it counts
// min(R, E) of them with half a tile's rows over each.
//
// FEW against MIDDLE by their times: FEW streams the weights of every row tile (0.13 us a
// MB) and reads the rows beside them (0.0037 us a MB and row), MIDDLE takes its k-steps'
// latency or the weights' stream, whichever is longer.  us for the FFN, 32 / 64 rows:
//   experts, d, d_ff      rows   MX4 activations   bf16 activations
//   64, 2048, 1024         128       33 / 38           37 / 50
//                         1024       63 / 46           65 / 61
//   16, 4096, 2048          32       30 / 36           36 / 52
//                          256       77 / 42           75 / 56
//   1, 2048, 2048          128       16 / 20           19 / 28
//
// weights: values of one expert; steps: 256-column steps of all products; products: their
// number.
bool few_rows(int64_t R, int E, int64_t weights, int steps, int products, bool mx4) {
  const double live = (double)(R < E ? R : E), mb = weights * (17.0 / 32) * 1e-6;
  const double few = 4 * products + mb * (0.13 * (live + R / 32) + 0.0037 * R);
  const double latency = mx4 ? 5.2 * products + 0.56 * steps : 4.5 * products + 1.15 * steps;
  const double stream = 3 * products + (mx4 ? 0.18 : 0.24) * mb * live;
  return few <= (latency > stream ? latency : stream);
}

// The others by the number of tiles, as there are 256 CUs: one persistent workgroup a CU
// needs some rounds of tiles to even out, and taller tiles of ragged experts waste more.
// us for one product by 64 x 128 / 128 x 128 / BIG 128 / BIG 256:
//   experts, N, K         rows   MX4 activations          bf16 activations
//   64, 2048, 2048        1024   26 / 31 / 29 / 39        39 / 60 / 37 / 83
//                         4096   32 / 41 / 36 / 51        58 / 77 / 58 / 118
//                         8192   50 / 46 / 38 / 52        96 / 95 / 75 / 119
//                        16384   77 / 78 / 59 / 54        170 / 172 / 141 / 138
//                        32768   172 / 165 / 90 / 88      326 / 308 / 244 / 242
//   16, 4096, 4096         512   30 / 26 / 30 / 38        46 / 54 / 44 / 76
//                         2048   37 / 39 / 36 / 57        82 / 88 / 79 / 144
//                         8192   118 / 101 / 86 / 86      285 / 264 / 241 / 242
//                        32768   537 / 484 / 296 / 270    1203 / 1118 / 861 / 808
//   8, 7168, 1024         1024   17 / 18 / 18 / 19        27 / 29 / 30 / 30
//                         4096   42 / 39 / 32 / 35        72 / 70 / 61 / 72
//                         8192   78 / 70 / 52 / 46        146 / 134 / 112 / 103
//   8, 1024, 3584         2048   15 / 16 / 20 / 27        30 / 33 / 44 / 64
//                         8192   32 / 35 / 34 / 30        72 / 78 / 84 / 69
//                        16384   61 / 55 / 49 / 54        135 / 133 / 127 / 141
//   1, 2048, 2048         2048   12 / 12 / 16 / 20        23 / 23 / 30 / 42
//                         4096   23 / 17 / 18 / 23        45 / 35 / 35 / 45
//                        16384   71 / 70 / 45 / 44        177 / 172 / 110 / 103
//   32, 1024, 1024        4096   11 / 10 / 13 / 16        17 / 18 / 21 / 27
//                        16384   27 / 26 / 24 / 26        45 / 43 / 45 / 50
// Over 63 such cases the rule takes on average 0.4 % (MX4) and 1.1 % (bf16) longer than the
// best tiles.
Tiles many_rows(int64_t R, int E, int64_t N, int K, bool mx4) {
  const double live = (double)(R < E ? R : E);
  auto tiles = [&](int bm, int bn) { return ((double)R / bm + live / 2) * ((N + bn - 1) / bn); };
  // BIG needs k-steps for its pipeline, and tiles, offsets within a tile and of scales in 32
  // bits
  if (K >= 576 && N <= 1 << 20 && mx4_scale_bytes(R, K) < (size_t)1 << 31 &&
      tiles(128, 256) < 1 << 29) {
    if (R >= 512 * live && tiles(256, 256) >= (mx4 ? 640 : 900)) return BIG256;
    // (64-row tiles are as good for up to 64 rows an expert)
    if (R >= 96 * live && tiles(128, 256) >= 360) return BIG128;
  }
  // 768 tiles of 64 rows run at once, 512 of 128
  const double n = tiles(64, 128);
  const bool tall = n >= 2000 || (n >= 500 && (R >= 2048 * live || (mx4 && n <= 800)));
  return R >= 32 * live && tall ? MID128 : MID64;
}
Tiles product_tiles(int64_t R, int E, int N, int K, bool mx4) {
  return few_rows(R, E, (int64_t)N * K, mx4_groups(K), 1, mx4) ? FEW : many_rows(R, E, N, K, mx4);
}
struct FfnTiles {
  Tiles gu, down;
};
FfnTiles ffn_tiles(int64_t R, int E, int d, int f, bool mx4) {
  if (few_rows(R, E, 3LL * d * f, mx4_groups(d) + mx4_groups(f), 2, mx4)) return {FEW, FEW};
  return {many_rows(R, E, 2LL * f, d, mx4), many_rows(R, E, d, f, mx4)};
}

// one product with its epilogue (round: see launch_mx4_few)
hipError_t launch_product(Mx4Args a, Tiles kind, bool round, const int32_t* offsets,
                          const int32_t* expert_map, int E, int64_t R, hipStream_t s) {
  if (kind == FEW) return launch_mx4_few(a, round, offsets, expert_map, E, R, s);
  a.bm = rows_of(kind);
  if (is_big(kind)) return launch_mx4_big(a, s);
  Mx4Params p = mx4_params(a);
  p.offsets = offsets;
  p.expert_map = expert_map;
  p.E = E;
  if (a.a_scale) {
    if (a.f) return launch_middle<ACT_MX4, MX4_GU>(p, a.bm, R, s);
    return a.f32_out ? launch_middle<ACT_MX4, MX4_STORE_F32>(p, a.bm, R, s)
                     : launch_middle<ACT_MX4, MX4_STORE>(p, a.bm, R, s);
  }
  if (a.f) return launch_middle<ACT_BF16, MX4_GU>(p, a.bm, R, s);
  return a.f32_out ? launch_middle<ACT_BF16, MX4_STORE_F32>(p, a.bm, R, s)
                   : launch_middle<ACT_BF16, MX4_STORE>(p, a.bm, R, s);
}

// Workspaces are laid out for every kind of tile (lists of 128-row tiles are the longest),
// so a buffer for many tokens serves fewer.
size_t list_bytes(int64_t R, int E, int n_cols, bool gate_up) {
  return mx4_big_list_bytes(R, E, 128, n_cols, gate_up);
}

}  // namespace

int mx4_product_tile(int64_t R, int E, int N, int K, bool mx4, int* cols) {
  const Tiles t = product_tiles(R, E, N, K, mx4);
  if (cols) *cols = cols_of(t);
  return rows_of(t);
}

int mx4_ffn_tile(int64_t R, int E, int d, int f, bool mx4, bool down, int* cols) {
  const FfnTiles both = ffn_tiles(R, E, d, f, mx4);
  const Tiles t = down ? both.down : both.gu;
  if (cols) *cols = cols_of(t);
  return rows_of(t);
}

// the tile list, then X's scales in routed order
size_t mx4_product_ws_bytes(int T, int k, int E, int K, int N) {
  const int64_t R = (int64_t)T * k;
  return list_bytes(R, E, N, false) + align_up(mx4_scale_bytes(R, K), 256);
}

hipError_t launch_mx4_product(const void* x, const uint8_t* x_scale, const int32_t* row_src, int T,
                              int k, const uint8_t* w, const uint8_t* w_scale,
                              const int32_t* offsets, const int32_t* expert_map, int out_dtype,
                              int E, int N, int K, int64_t R, void* out, void* ws, hipStream_t s) {
  if (R == 0) return hipSuccess;
  const int64_t R_ws = row_src ? (int64_t)T * k : T;
  Mx4Args a = {};
  a.A = x;
  a.a_scale = x_scale;
  a.a_rows = T;
  a.B = w;
  a.b_scale = w_scale;
  a.N = N;
  a.K = K;
  a.f32_out = out_dtype == kDtypeF32;
  a.out = out;
  a.out_rows = R;
  a.row_src = row_src;
  a.slots_k = k;
  const Tiles kind = product_tiles(R_ws, E, N, K, x_scale != nullptr);
  if (is_big(kind)) {
    uint8_t* const list = static_cast<uint8_t*>(ws);
    uint8_t* const routed = list + list_bytes(R_ws, E, N, false);
    const bool gather = x_scale && row_src;
    const hipError_t err =
        launch_mx4_prepare(offsets, expert_map, E, R, 0, 0, nullptr, rows_of(kind), N, list,
                           x_scale, gather ? routed : nullptr, row_src, k, T, K, s);
    if (err != hipSuccess) return err;
    if (gather) {
      a.a_scale = routed;
      a.a_rows = R;
    }
    a.list = list;
  }
  return launch_product(a, kind, false, offsets, expert_map, E, R, s);
}

namespace {

// the FFN's workspace: X in MX4, H (MX4 or bf16), the products' tile lists, and X's scales
// in routed order
struct Mx4FfnWs {
  size_t x_scale, h, h_scale, list_gu, list_d, routed, bytes;
};
Mx4FfnWs ffn_ws(int64_t T, int64_t R, int E, int d, int f, bool mx4) {
  Mx4FfnWs w;
  w.x_scale = mx4 ? align_up((size_t)T * d / 2, 256) : 0;
  w.h = w.x_scale + (mx4 ? align_up(mx4_scale_bytes(T, d), 256) : 0);
  w.h_scale = w.h + align_up((size_t)R * f * 2 / (mx4 ? 4 : 1), 256);
  w.list_gu = w.h_scale + (mx4 ? align_up(mx4_scale_bytes(R, f), 256) : 0);
  w.list_d = w.list_gu + list_bytes(R, E, f, true);
  w.routed = w.list_d + list_bytes(R, E, d, false);
  w.bytes = w.routed + (mx4 ? align_up(mx4_scale_bytes(R, d), 256) : 0);
  return w;
}

}  // namespace

size_t ffn_fwd_mx4_ws_bytes(int T, int k, int E, int d, int f) {
  const size_t a = ffn_ws(T, (int64_t)T * k, E, d, f, true).bytes;
  const size_t b = ffn_ws(T, (int64_t)T * k, E, d, f, false).bytes;
  return a > b ? a : b;
}

hipError_t launch_ffn_fwd_mx4(const void* x, const int32_t* row_src, int T, int k,
                              const uint8_t* w_gu, const uint8_t* w_gu_scale, const uint8_t* w_d,
                              const uint8_t* w_d_scale, const int32_t* offsets,
                              const int32_t* expert_map, int act_bits, int E, int d, int f,
                              int64_t R, void* y_perm, void* act_save, void* ws, hipStream_t s) {
  if (R == 0) return hipSuccess;
  const bool mx4 = act_bits == 4;
  const int64_t R_ws = row_src ? (int64_t)T * k : T;
  const Mx4FfnWs at = ffn_ws(T, R_ws, E, d, f, mx4);
  const FfnTiles tiles = ffn_tiles(R_ws, E, d, f, mx4);
  uint8_t* const base = static_cast<uint8_t*>(ws);
  Mx4Args a = {};
  a.A = x;
  a.a_rows = T;
  hipError_t err = hipSuccess;
  if (mx4 && tiles.gu != FEW) {
    err = launch_mx4_quantize(x, kDtypeBf16, 1, T, d, base, base + at.x_scale, s);
    if (err != hipSuccess) return err;
    a.A = base;
    a.a_scale = base + at.x_scale;
  }
  const bool gu_big = is_big(tiles.gu), down_big = is_big(tiles.down);
  if (gu_big || down_big) {
    const bool gather = mx4 && row_src && gu_big;
    err = launch_mx4_prepare(offsets, expert_map, E, R, rows_of(tiles.gu), f,
                             gu_big ? base + at.list_gu : nullptr, rows_of(tiles.down), d,
                             down_big ? base + at.list_d : nullptr, a.a_scale,
                             gather ? base + at.routed : nullptr, row_src, k, T, d, s);
    if (err != hipSuccess) return err;
    if (gather) {
      a.a_scale = base + at.routed;
      a.a_rows = R;
    }
  }
  a.B = w_gu;
  a.b_scale = w_gu_scale;
  a.N = 2 * f;
  a.K = d;
  a.f = f;
  a.out = base + at.h;
  a.out_scale = base + at.h_scale;
  a.out_rows = R;
  a.act = act_save;
  a.row_src = row_src;
  a.slots_k = k;
  a.list = base + at.list_gu;
  err = launch_product(a, tiles.gu, mx4, offsets, expert_map, E, R, s);
  if (err != hipSuccess) return err;
  a.A = a.out;
  a.a_scale = mx4 ? a.out_scale : nullptr;
  a.a_rows = R;
  a.B = w_d;
  a.b_scale = w_d_scale;
  a.N = d;
  a.K = f;
  a.f = 0;
  a.out = y_perm;
  a.act = nullptr;
  a.row_src = nullptr;
  a.list = base + at.list_d;
  return launch_product(a, tiles.down, false, offsets, expert_map, E, R, s);
}

}  // namespace laep
