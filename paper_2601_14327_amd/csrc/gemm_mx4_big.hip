// Grouped products at MX4 weights for many rows: the products of gemm_mx4.hip in tiles of
// 256 or 128 x 256, one persistent workgroup of eight waves (2 x 4, each 128 or 64 x 64) a
// CU.
//
// The k-steps of all the tiles that a workgroup walks are one stream: copies run two to
// four steps ahead of the matrix instructions, past a tile's end into the next tile, whose
// token rows were read a tile earlier, and so do the reads of fragments.  A tile's epilogue,
// from registers to memory, lies between two steps with the next tile's operands landed or
// in flight.  Rings in the LDS, and what a step is:
//   MX4, 256 rows:   256 columns; three slots of A (32 KB), two of B, whose fragments are
//                    all in registers after a quarter of the step.  Scales go to registers,
//                    a dword per fragment and step, as the LDS is full, in two sets.  The
//                    compiler copies one of them at the loop's head, where every second
//                    step so waits for scales that it loaded itself, and for the copies of
//                    A before them.
//   MX4, 128 rows:   256 columns; three slots of A (16 KB), of B and of scales.
//   bf16, 256 rows:  64 columns; four slots of A (32 KB) and of weight codes (8 KB).
//   bf16, 128 rows:  64 columns; five slots of A (16 KB), two of the codes and scales of four
//                    steps: 128 bytes of a row, a whole line (by 32 bytes each line crosses
//                    from L2 four times: 0.80 us a step of one 32-row block, 0.43 so).
// Scales of gathered MX4 activations lie in routed order (that of a gathered row would cost
// a cache line a step, as much as its codes).
//
// In 128-row tiles a wave leaves out 32-row blocks without rows, so ragged experts cost what
// their rows do: such tiles are dealt tallest first, forward and back (64 experts of 128
// rows on average, 2048 x 2048, bf16: 95 -> 81 us).
//
// Measured on products of 64 even experts, 2048 x 2048, lists included: 256-row tiles of
// 1024 and 2048 rows an expert in MX4 159 and 301 us (3.5 and 3.6 PFLOP/s), in bf16 417 and
// 810 (1.32 and 1.36; a large library product: 1.60), with uneven experts the matrix cores
// are busy 44 and 62 - 67 % of the cycles; 128-row tiles of 128 and 256 rows in MX4 35 and 48, in bf16 64 and 111
// (1.08 and 1.24 PFLOP/s).  Where weights are hardly shared (up to 128 rows an expert) the
// weights' stream bounds: 142 MB of codes and scales in MX4's 35 us.
//
// The 256-row bf16 SwiGLU kernel keeps 15 registers in scratch, some of them for the kept
// pre-activations' path, and reloads them where the next tile's rows are read, where the
// copies move on to it, and after a tile's stores: there it waits for everything in flight.
#include <type_traits>

#include "gemm_mx4.hpp"

namespace laep {
namespace {

constexpr int kBigThreads = 512;
constexpr int kBigBN = 256;

// The tile list holds the tiles by classes of height, the tallest first; their starts, and
// the end, lie kClassOffset ints into its header.
constexpr int kClasses = 4, kClassOffset = 32;

struct BigTile {
  int row0, rows, phys, nt;
};

// H in MX4 needs a row's columns in one lane (its blocks' largest magnitudes); the other
// outputs take the columns along the lanes, so that a store covers whole lines of a row.
template <int ACT, int EPI>
constexpr bool rows_in_lanes() { return EPI == MX4_GU && ACT == ACT_MX4; }

// stores of one 32-row block of a wave's tile
template <int ACT, int EPI>
constexpr int block_stores() {
  return EPI != MX4_GU ? 16 : ACT == ACT_MX4 ? 2 : 8;
}

// Two rows of one column in every lane (low half: row r, high half: row r + 1) become two
// columns of one row: an even lane ends up with columns (c, c + 1) of row r, the odd lane
// beside it with the same columns of row r + 1.
__device__ __forceinline__ uint32_t column_pair(uint32_t v, int lane) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
  return __builtin_amdgcn_perm(o, v, lane & 1 ? 0x03020706u : 0x05040100u);
}

// One 32-row block of a wave.  Rows in lanes: acc[j][4q + i] is row lane % 32, column 8q + 4
// (lane / 32) + i of fragment j.  Columns in lanes: row 8q + 4 (lane / 32) + i, column
// lane % 32.  Descriptors end with the tile's rows: stores past them, or at dropped
// offsets, write nothing, and every wave issues the same number.
template <int ACT, int EPI, int WTM>
__device__ __forceinline__ void store_block(const Mx4Params& p, const BigTile& te, int i, int wm,
                                            int wn, int lane, const f32x16_t acc[2]) {
  const int half = lane >> 5;
  auto rsrc_of = [&](void* base, long long bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(base, 0, (int)bytes, kBufferFlags);
  };
  const uint32_t row0 = wm * WTM + i * 32;
  if constexpr (EPI == MX4_GU) {
    const int f = p.f, fcol = te.nt * 128 + wn * 32;   // f % 64 == 0: whole blocks
    const bool in = fcol < f;
    float h[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) h[r] = fast_silu(acc[0][r]) * acc[1][r];
    if constexpr (ACT == ACT_MX4) {
      const uint32_t row = row0 + (lane & 31);
      u32x2_t w;
      const uint32_t b = mx4_row_block(h, w);
      const __amdgpu_buffer_rsrc_t rc = rsrc_of(
          static_cast<char*>(p.out) + (long long)te.row0 * (f / 2), (long long)te.rows * (f / 2));
      const __amdgpu_buffer_rsrc_t rs =
          rsrc_of(p.out_scale + ((long long)(fcol / kMx4Group) * p.out_rows + te.row0) * 8,
                  in ? te.rows * 8 : 0);
      __builtin_amdgcn_raw_buffer_store_b64(
          w, rc, in ? (int)(row * (f / 2) + fcol / 2 + half * 8) : (int)kDroppedCopy, 0, 0);
      const uint32_t at = half ? kDroppedCopy : row * 8;
      __builtin_amdgcn_raw_buffer_store_b8((uint8_t)b, rs, (int)at, fcol / kMx4Block % 8, 0);
      if (fcol + kMx4Block == f)   // the blocks past f
        for (int k = f / kMx4Block; k % 8; ++k)
          __builtin_amdgcn_raw_buffer_store_b8((uint8_t)0, rs, (int)at, k % 8, 0);
    } else {
      const uint32_t row = row0 + 4 * half + (lane & 1), col = fcol + (lane & 30);
      if (p.act) {
        const __amdgpu_buffer_rsrc_t ra =
            rsrc_of(p.act + (long long)te.row0 * 2 * f, (long long)te.rows * 4 * f);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            const uint32_t at = in ? ((row + 8 * q + r) * 2 * f + col) * 2 : kDroppedCopy;
            const uint32_t up = in ? at + 2 * f : kDroppedCopy;
            const int e = 4 * q + r;
            __builtin_amdgcn_raw_buffer_store_b32(
                column_pair(pack_bf16x2(acc[0][e], acc[0][e + 1]), lane), ra, (int)at, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b32(
                column_pair(pack_bf16x2(acc[1][e], acc[1][e + 1]), lane), ra, (int)up, 0, 0);
          }
      }
      const __amdgpu_buffer_rsrc_t rh = rsrc_of(
          static_cast<bf16_t*>(p.out) + (long long)te.row0 * f, (long long)te.rows * 2 * f);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int r = 0; r < 4; r += 2)
          __builtin_amdgcn_raw_buffer_store_b32(
              column_pair(pack_bf16x2(h[4 * q + r], h[4 * q + r + 1]), lane), rh,
              in ? (int)(((row + 8 * q + r) * f + col) * 2) : (int)kDroppedCopy, 0, 0);
    }
  } else {
    // fragments 0 and 1 hold the even and odd ones of the wave's 64 columns
    constexpr int ES = EPI == MX4_STORE ? 2 : 4;
    const __amdgpu_buffer_rsrc_t ro = rsrc_of(
        static_cast<char*>(p.out) + (long long)te.row0 * p.N * ES, (long long)te.rows * p.N * ES);
    const int c0 = te.nt * 256 + wn * 64;              // N % 64 == 0: a wave's columns are whole
    const uint32_t ld = (uint32_t)p.N * ES;
    const uint32_t at = c0 < p.N ? (row0 + 4 * half) * ld + (c0 + 2 * (lane & 31)) * ES : kDroppedCopy;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t o = at + (q * 8 + r) * ld;
        if constexpr (EPI == MX4_STORE)
          __builtin_amdgcn_raw_buffer_store_b32(pack_bf16x2(acc[0][4 * q + r], acc[1][4 * q + r]),
                                                ro, (int)o, 0, kDmaStream);
        else
          __builtin_amdgcn_raw_buffer_store_b64(
              u32x2_t{__float_as_uint(acc[0][4 * q + r]), __float_as_uint(acc[1][4 * q + r])}, ro,
              (int)o, 0, kDmaStream);
      }
  }
}

template <int ACT, int EPI, int BM>
__global__ __launch_bounds__(kBigThreads) void gemm_mx4_big_kernel(Mx4Params p) {
  constexpr bool MX4 = ACT == ACT_MX4;
  constexpr int NT = kBigThreads, WTM = BM / 2, TM = WTM / 32, TN = 2;
  // bf16, 128 rows: weights by groups of four steps
  constexpr bool GROUPED = !MX4 && BM == 128;
  // scales through the LDS (256 rows leave no room there: in registers)
  constexpr bool LDS_SCALES = BM == 128;
  constexpr int APART = BM * 128;                    // a step's activations
  constexpr int BPART = MX4 || GROUPED ? kBigBN * 128 : kBigBN * 32;   // its (a group's) weights
  // steps in the LDS: of A; of B (256 rows in MX4: one fewer; or groups)
  constexpr int NSLOT = MX4 ? 3 : GROUPED ? 5 : 4;
  constexpr int NSLOTB = GROUPED || (MX4 && BM == 256) ? 2 : NSLOT;
  constexpr int AHEAD = MX4 ? 2 : NSLOT - 1;         // steps the copies run ahead
  constexpr int NH = APART / 16 / NT;                // copies a thread and step of A
  constexpr int NB = BPART / 16 / NT;                // and of B (a group: one a step)
  static_assert(BM == 256 || BM == 128, "two rows of waves");
  // Scales of a step or group, two dwords a thread.  Bf16: those of the wave's own 64 weight
  // rows.  MX4: low and high dwords of 256 weight rows, of 128 rows of A, and 1 KB not used.
  constexpr int SPART = LDS_SCALES ? NT * 8 : 0;
  constexpr int SMEM = NSLOT * APART + NSLOTB * (BPART + SPART);
  static_assert(SMEM <= 160 * 1024, "the LDS");
  __shared__ __attribute__((aligned(1024))) char smem[SMEM];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5;
  const int wm = wave / 4, wn = wave % 4;
  // this XCD's part of every class of the tile list (block i runs on XCD i % 8), dealt to
  // its workgroups in turn, forward and back: the tallest tiles first
  const int stride = gridDim.x >> 3, slot = blockIdx.x >> 3;
  int class_lo[kClasses], class_n[kClasses], n_tiles = 0;
#pragma unroll
  for (int c = 0; c < kClasses; ++c) {
    const int lo = p.n_entries[kClassOffset + c], n = p.n_entries[kClassOffset + c + 1] - lo;
    class_lo[c] = lo + (int)((long long)n * (blockIdx.x & 7) / 8);
    class_n[c] = lo + (int)((long long)n * ((blockIdx.x & 7) + 1) / 8) - class_lo[c];
    n_tiles += class_n[c];
  }
  int round = 0;
  auto tile_of = [&](int r) { return r * stride + (BM == 128 && r & 1 ? stride - 1 - slot : slot); };
  if (tile_of(0) >= n_tiles) return;

  auto load_entry = [&](int q) {   // through the scalar cache
    int at = 0;
#pragma unroll
    for (int c = 0; c < kClasses; ++c) {
      if (q >= 0 && q < class_n[c]) at = class_lo[c] + q;
      q -= class_n[c];
    }
    const auto* t = (const __attribute__((address_space(4))) int*)(uintptr_t)(p.table + at);
    BigTile e;
    e.row0 = t[0];
    e.rows = t[1];
    e.phys = t[3];
    e.nt = t[4];
    return e;
  };
  auto weight_row = [&](int nt, int r) {
    if (EPI == MX4_GU) {   // per 64: 32 gate rows, then the same columns' up rows
      int fcol = nt * 128 + (r >> 6) * 32 + (r & 31);
      fcol = fcol < p.f ? fcol : p.f - 1;
      return r & 32 ? p.f + fcol : fcol;
    }
    // per 64: the even columns, then the odd ones
    const int row = nt * 256 + (r & ~63) + 2 * (r & 31) + (r >> 5 & 1);
    return row < p.N ? row : p.N - 1;
  };
  const int a_row_bytes = MX4 ? p.K / 2 : p.K * 2;
  const int G = (p.K + kMx4Group - 1) / kMx4Group;
  const int nk = MX4 ? G : p.K / 64;                 // (host: at least 3, bf16 9)

  // ---- copies: rows of the next tile, then offsets and descriptors of the tile that is
  // being copied, which the end of its last step moves on
  uint32_t raw[NH];
  auto load_rows = [&](const BigTile& t) {
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const int r = (i * NT + tid) >> 3;
      const int rr = r < t.rows ? r : t.rows - 1;
      raw[i] = p.row_src ? (uint32_t)p.row_src[t.row0 + rr] : (uint32_t)rr;
    }
  };
  uint32_t a_voff[NH], b_voff;
  int b_group[NB];                                   // byte offsets of 64 rows each
  uint32_t s_voff, sa_voff = kDroppedCopy;
  __amdgpu_buffer_rsrc_t s_rsrc, sa_rsrc;
  __amdgpu_buffer_rsrc_t a_rsrc, b_rsrc;
  int c_step = 0;                                    // step of its tile that is copied next
  const int a_lc = (tid & 7) ^ swz8(tid >> 3);       // chunk of a row (64 rows on: the same)
  // The rows' offsets, once loaded (no tile left: the copies are dropped; so are those of
  // rows past the tile's end: zeros, at which the matrix cores draw less power than at
  // another row's values).
  auto finish_rows = [&](const BigTile& t, bool left) {
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const uint32_t row = p.row_src ? raw[i] / (uint32_t)p.slots_k : raw[i];
      const bool in = left && ((i * NT + tid) >> 3) < t.rows;
      raw[i] = in ? row * (uint32_t)a_row_bytes + a_lc * 16 : kDroppedCopy;
    }
  };
  auto begin_a = [&](const BigTile& t) {
    const long long row0 = p.row_src ? 0 : t.row0;
#pragma unroll
    for (int i = 0; i < NH; ++i) a_voff[i] = raw[i];
    a_rsrc = mx4_rsrc(static_cast<const char*>(p.A) + row0 * a_row_bytes);
    c_step = 0;
  };
  auto a_scales_of = [&](const BigTile& t) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(p.a_scale) + (long long)t.row0 * 8, 0,
        (int)((G * p.a_rows - t.row0) * 8), kBufferFlags);
  };
  int c_group = 0;                                   // (grouped) the weights' group, likewise
  auto begin_b = [&](const BigTile& t, bool left) {
    // 64 rows of the tile lie in the matrix or past it (f and N are multiples of 64: past
    // it, the first 64 again); bf16 by steps: two chunks a row, rows 4 apart swap them
    constexpr bool WIDE = MX4 || GROUPED;
    const int r = WIDE ? tid >> 3 : tid >> 1;
    const int lc = WIDE ? a_lc : (tid & 1) ^ ((r >> 2) & 1);
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int at = EPI == MX4_GU ? 32 * i : 64 * i;
        const bool in = EPI == MX4_GU ? t.nt * 128 + at < p.f : t.nt * 256 + at < p.N;
        b_group[i] = in ? at * (p.K / 2) : 0;
      }
    }
    b_voff = left ? (uint32_t)weight_row(t.nt, r) * (uint32_t)(p.K / 2) + lc * 16 : kDroppedCopy;
    b_rsrc = mx4_rsrc(p.B + (long long)t.phys * p.N * (p.K / 2));
    if constexpr (LDS_SCALES) {
      s_voff = left ? (uint32_t)weight_row(t.nt, wn * 64 + lane) * 8 + (MX4 ? wm * 4 : 0)
                    : kDroppedCopy;
      s_rsrc = mx4_rsrc(p.b_scale + (long long)t.phys * G * p.N * 8);
      c_group = 0;
    }
    if constexpr (LDS_SCALES && MX4) {
      // rows past the tile's end take other rows' scales, past the array's end none
      if (left && wave < 4) sa_voff = ((wave & 1) * 64 + lane) * 8 + (wave >> 1) * 4;
      else sa_voff = kDroppedCopy;
      sa_rsrc = a_scales_of(t);
    }
  };
  auto begin_copies = [&](const BigTile& t, bool left) {
    begin_a(t);
    begin_b(t, left);
  };
  // the columns of the last, partial 256 that lie past K are dropped
  auto codes_at = [&](uint32_t voff, int group) {
    return group * kMx4Group + a_lc * kMx4Block < p.K ? voff : kDroppedCopy;
  };
  int a_slot = 0, b_slot = 0;
  auto copy_a = [&](int i) {
    char* const dst = smem + a_slot * APART + i * NT * 16;
    uint32_t v[1] = {a_voff[i]};
    if constexpr (MX4) v[0] = codes_at(v[0], c_step);
    if constexpr (GROUPED) v[0] = c_step * 64 < p.K ? v[0] : kDroppedCopy;
    dma_chunks<1, NT>(dst, a_rsrc, v, c_step * 128, wave);
  };
  auto copy_b = [&](int i) {
    char* const dst = smem + NSLOT * APART + b_slot * BPART + i * NT * 16;
    const int g = GROUPED ? c_group : c_step;
    const uint32_t v[1] = {MX4 || GROUPED ? codes_at(b_voff, g) : b_voff};
    dma_chunks<1, NT>(dst, b_rsrc, v, MX4 || GROUPED ? b_group[i] + g * 128 : g * 32, wave);
  };
  auto scales_at = [&](int slot) { return smem + NSLOT * APART + NSLOTB * BPART + slot * SPART; };
  auto copy_s = [&](int h) {                         // (bf16: to wave * 512 + h * 256)
    if constexpr (!MX4)
      dma_scales(scales_at(b_slot) + wave * 256 + h * 256, s_rsrc, s_voff,
                 c_group * p.N * 8 + h * 4, wave);
    else if (h == 0)
      dma_scales(scales_at(b_slot), s_rsrc, s_voff, c_step * p.N * 8, wave);
    else
      dma_scales(scales_at(b_slot) + 2048, sa_rsrc, sa_voff, (int)(c_step * p.a_rows * 8), wave);
  };
  auto copied_b = [&]() {
    b_slot = b_slot + 1 == NSLOTB ? 0 : b_slot + 1;
    ++c_group;
  };
  auto copied = [&]() {                              // both operands of a step are issued
    ++c_step;
    a_slot = a_slot + 1 == NSLOT ? 0 : a_slot + 1;
    if constexpr (!GROUPED) b_slot = b_slot + 1 == NSLOTB ? 0 : b_slot + 1;
  };

  // ---- scales of a step: a dword per fragment (MX4: two steps ahead, in two sets), or
  // the byte of the lane's block (bf16)
  constexpr int NSET = MX4 ? 2 : 1;
  uint32_t sa[TM], sb[TN], sa_next[NSET][TM], sb_next[NSET][TN], sa_off, sb_off;
  int sb_far;                                        // from fragment 0's scales to 1's
  __amdgpu_buffer_rsrc_t sb_rsrc;
  auto begin_scales = [&](const BigTile& t) {
    if constexpr (MX4) {
      // rows past the tile's end take other rows' scales, past the array's end none
      sa_off = (wm * WTM + (lane & 31)) * 8 + half * 4;
      sa_rsrc = a_scales_of(t);
    }
    // fragment 1: the up rows, or the odd columns
    sb_off = weight_row(t.nt, wn * 64 + (lane & 31)) * 8 + half * (MX4 ? 4 : 1);
    sb_far = EPI == MX4_GU ? p.f * 8 : 8;
    sb_rsrc = mx4_rsrc(p.b_scale + (long long)t.phys * G * p.N * 8);
  };
  constexpr int NS = LDS_SCALES ? 2 : MX4 ? TM + TN : TN;
  auto load_scale = [&](int set, int n, int step) {
    if constexpr (MX4) {
      if (n < TN)
        sb_next[set][n] = __builtin_amdgcn_raw_buffer_load_b32(
            sb_rsrc, sb_off, step * p.N * 8 + n * sb_far, 0);
      else
        sa_next[set][n - TN] = __builtin_amdgcn_raw_buffer_load_b32(
            sa_rsrc, sa_off + (n - TN) * 256, (int)(step * p.a_rows * 8), 0);
    } else {
      sb_next[set][n] = __builtin_amdgcn_raw_buffer_load_b8(
          sb_rsrc, sb_off, (step >> 2) * p.N * 8 + 2 * (step & 3) + n * sb_far, 0);
    }
  };
  auto take_scales = [&](int set) {
    if constexpr (MX4) {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = sa_next[set][i];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j)
      sb[j] = MX4 ? sb_next[set][j] : __float_as_uint(mx4_scale(sb_next[set][j]));
  };

  // ---- fragments: sub-step s of a step at ^ 16 s; bf16 weights once a step
  // (64 rows on the swizzle is the same: fragments 2 and 3 at + 8 KB)
  int a_off[2], b_off[TN];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = wm * WTM + i * 32 + (lane & 31);
    a_off[i] = r * 128 + (((4 * half) ^ swz8(r)) << 4);
  }
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int r = wn * 64 + j * 32 + (lane & 31);
    b_off[j] = MX4       ? r * 128 + (((4 * half) ^ swz8(r)) << 4)
               : GROUPED ? r * 128 + ((half ^ swz8(r)) << 4)
                         : r * 32 + ((half ^ ((r >> 2) & 1)) << 4);
  }
  f32x16_t acc[TM][TN];
  auto zero_acc = [&]() {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  };
  u32x4_t fa0[TM], fa1[TM];                          // A of a sub-step and of the next
  u32x4_t fb[MX4 || GROUPED ? 4 : 1][TN];            // MX4: a step's B whole; bf16: its codes
  int ra = 0, rb = 0;                                // slots that are read
  auto a_base = [&]() { return smem + ra * APART; };
  auto b_base = [&]() { return smem + NSLOT * APART + rb * BPART; };
  auto read_a = [&](u32x4_t* ga, int s, int i) {
    ga[i] = *reinterpret_cast<const u32x4_t*>(a_base() + (a_off[i & 1] ^ (s << 4)) + (i >> 1) * 8192);
  };
  auto read_b = [&](int s, int j) {
    fb[s][j] = *reinterpret_cast<const u32x4_t*>(b_base() + (b_off[j] ^ (s << (GROUPED ? 5 : 4))));
  };
  // (MX4) a fragment's scales from the LDS, of the step to come
  auto read_s4 = [&](int n) {
    const char* const at = scales_at(rb) + (n < TN ? half * 1024 + (wn * 64 + n * 32) * 4
                                                   : 2048 + half * 512 + (wm * WTM + (n - TN) * 32) * 4);
    const uint32_t v = *reinterpret_cast<const uint32_t*>(at + (lane & 31) * 4);
    if (n < TN) sb_next[0][n] = v;
    else sa_next[0][n - TN] = v;
  };
  // (grouped) the scales of a group: lane's fragments, dwords of blocks 0 - 3 and 4 - 7
  uint32_t raw_s[TN][2];
  auto read_s = [&](int j, int h) {
    raw_s[j][h] = *reinterpret_cast<const uint32_t*>(scales_at(rb) + wave * 512 + h * 256 +
                                                     (j * 32 + (lane & 31)) * 4);
  };
  auto to_numbers = [&](int q) {                     // those of step q of the group
#pragma unroll
    for (int j = 0; j < TN; ++j)
      sb[j] = __float_as_uint(mx4_scale((raw_s[j][q >> 1] >> (16 * (q & 1) + 8 * half)) & 255));
  };
  // Sub-step S on BLOCKS fragments of fa, beside its matrix instructions READS fragment
  // reads (of what later sub-steps take), and extra(n) at every EVERY-th of them, COUNT times.
  auto sub_step = [&](auto blocks_tag, auto s_tag, const u32x4_t* fa, const u32x4_t* w, auto reads_tag, auto read,
                      auto every_tag, auto count_tag, auto extra) __attribute__((always_inline)) {
    constexpr int S = decltype(s_tag)::value, EVERY = decltype(every_tag)::value;
    constexpr int COUNT = decltype(count_tag)::value, READS = decltype(reads_tag)::value;
    constexpr int NMM = decltype(blocks_tag)::value * TN, SLOTS = EVERY * COUNT;
    constexpr int WORK = NMM > READS ? NMM : READS, MOST = WORK > SLOTS ? WORK : SLOTS;
    u32x4_t wv[TN];
    if constexpr (!MX4 && NMM > 0) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
        wv[j] = mx4_values8_bf16(w[j][S], __uint_as_float(sb[j]));
    }
#pragma unroll
    for (int n = 0; n < MOST; ++n) {
      if (n < NMM) {
        const int i = n / TN, j = n % TN;
        if constexpr (rows_in_lanes<ACT, EPI>())
          acc[i][j] = mfma_mx4<S>(fb[S][j], fa[i], sb[j], sa[i], acc[i][j]);
        else if constexpr (MX4)
          acc[i][j] = mfma_mx4<S>(fa[i], fb[S][j], sa[i], sb[j], acc[i][j]);
        else
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8_t, fa[i]), __builtin_bit_cast(bf16x8_t, wv[j]), acc[i][j],
              0, 0, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      }
      if (n < READS) {
        read(n);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      if (n < SLOTS && n % EVERY == EVERY - 1) {
        extra(n / EVERY);
        __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);   // nothing moves between sub-steps
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  using I2 = std::integral_constant<int, 2>;
  using I3 = std::integral_constant<int, 3>;
  using CopiesA = std::integral_constant<int, NH>;
  using CopiesB = std::integral_constant<int, NB>;
  using All = std::integral_constant<int, TM>;
  using Scales = std::integral_constant<int, NS>;
  auto nothing = [](int) {};

  // ---- the stream
  BigTile cur = load_entry(tile_of(0)), nxt = cur;
  load_rows(cur);
  finish_rows(cur, true);
  begin_copies(cur, true);
  if constexpr (!LDS_SCALES) begin_scales(cur);
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
#pragma unroll
    for (int i = 0; i < NH; ++i) copy_a(i);
    if (!GROUPED || t < NSLOTB) {
#pragma unroll
      for (int i = 0; i < NB; ++i) copy_b(i);
    }
    if (LDS_SCALES && (MX4 || t < NSLOTB)) {
      copy_s(0);
      copy_s(1);
      if constexpr (GROUPED) copied_b();
    }
    copied();
  }
  if constexpr (MX4) {                               // (A runs one step further ahead)
#pragma unroll
    for (int i = 0; i < NH; ++i) copy_a(i);
  }
#pragma unroll
  for (int t = 0; t < (LDS_SCALES ? 0 : NSET); ++t)
#pragma unroll
    for (int n = 0; n < NS; ++n) load_scale(t, n, t);
  round = 1;
  bool more = tile_of(1) < n_tiles;
  if (more) {
    nxt = load_entry(tile_of(1));
    load_rows(nxt);
  }
  wait_vmcnt<0>();                                   // (once a workgroup)
  finish_rows(nxt, more);
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < TM; ++i) read_a(fa0, 0, i);
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int s = 0; s < (MX4 ? 3 : 1); ++s) read_b(s, j);
  if constexpr (MX4 && LDS_SCALES) {
#pragma unroll
    for (int n = 0; n < TM + TN; ++n) read_s4(n);
  }
  if constexpr (GROUPED) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) read_s(j, h);
    to_numbers(0);
  } else if constexpr (!MX4) {
    take_scales(0);
  }
  constexpr int S_ALL = TM * block_stores<ACT, EPI>();
  // the matrix instructions stay where they are, and what is derived from the fragments'
  // offsets is not kept
  auto fence = [&]() {
#pragma unroll
    for (int i = 0; i < TM; ++i) opaque(acc[i][0], acc[i][1]);
    opaque(a_off[0], a_off[1]);
    opaque(b_off[0], b_off[1]);
  };
  // MX4: the last sub-step of a step, after the barrier that ends it: beside it the reads
  // of the next step's first fragments (those of NEXT blocks), and the copies of A two steps
  // past that one into the slot that the step has just freed.
  auto last_sub = [&](auto blocks, auto next_tag) __attribute__((always_inline)) {
    constexpr int NEXT = decltype(next_tag)::value;
    constexpr int SC = LDS_SCALES && NEXT ? TM + TN : 0;
    sub_step(blocks, I3{}, fa1, fb[0], std::integral_constant<int, NEXT ? NEXT + 3 * TN + SC : 0>{},
             [&](int n) {
      if (n < TN) read_b(0, n);
      else if (n < TN + NEXT) read_a(fa0, 0, n - TN);
      else if (n < TN + NEXT + SC) read_s4(n - TN - NEXT);
      else read_b(1 + (n - TN - NEXT - SC) / TN, (n - TN - NEXT - SC) % TN);
    }, I1{}, CopiesA{}, [&](int n) { copy_a(n); });
    fence();
  };
  // MX4: the rest of a step.  Its B fragments are all in registers after the first
  // sub-step, so that B's slot is free for the copies of two steps on.
  auto first_subs = [&](auto blocks, auto early_tag, auto set_tag, int s_step)
                        __attribute__((always_inline)) {
    constexpr bool EARLY = decltype(early_tag)::value;
    constexpr int SET = decltype(set_tag)::value, BLOCKS = decltype(blocks)::value;
    take_scales(SET);
    sub_step(blocks, I0{}, fa0, fb[0], std::integral_constant<int, BLOCKS ? BLOCKS + TN : 0>{}, [&](int n) {
      if (n < BLOCKS) read_a(fa1, 1, n);
      else read_b(3, n - BLOCKS);
    }, I1{}, std::integral_constant<int, LDS_SCALES ? 0 : NS>{},
             [&](int n) { load_scale(SET, n, s_step); });
    if constexpr (NSLOTB == 2) {                     // (with three slots B's is free already)
      wait_lgkm0();
      __builtin_amdgcn_s_barrier();
    }
    sub_step(blocks, I1{}, fa1, fb[0], blocks, [&](int n) { read_a(fa0, 2, n); },
             std::integral_constant<int, TM / 2>{}, std::integral_constant<int, NB + (LDS_SCALES ? 2 : 0)>{},
             [&](int n) {
      if (n < NB) copy_b(n);
      else copy_s(n - NB);
    });
    copied();
    sub_step(blocks, I2{}, fa0, fb[0], blocks, [&](int n) { read_a(fa1, 3, n); }, I1{}, I0{}, nothing);
    // The next step has landed: after its copies (of B in the step before this) came A's
    // and B's of two steps on, six scales and, in a tile's first step, the stores of the
    // tile before.
    constexpr int W = NH + NB + NS + (EARLY ? S_ALL : 0);
    wait_vmcnt_lgkm0<(W < 63 ? W : 63)>();
    __builtin_amdgcn_s_barrier();
    ra = ra + 1 == NSLOT ? 0 : ra + 1;
    rb = rb + 1 == NSLOTB ? 0 : rb + 1;
    fence();
  };
  // bf16: one step; EARLY: the first AHEAD - 1 of a tile
  auto bf16_step = [&](auto blocks, auto next_tag, auto early_tag, int s_step)
                       __attribute__((always_inline)) {
    constexpr bool EARLY = decltype(early_tag)::value;
    sub_step(blocks, I0{}, fa0, fb[0], blocks, [&](int n) { read_a(fa1, 1, n); }, I1{}, Scales{},
             [&](int n) { load_scale(0, n, s_step); });
    sub_step(blocks, I1{}, fa1, fb[0], blocks, [&](int n) { read_a(fa0, 2, n); }, I2{}, CopiesA{},
             [&](int n) { copy_a(n); });
    sub_step(blocks, I2{}, fa0, fb[0], blocks, [&](int n) { read_a(fa1, 3, n); }, I1{}, CopiesB{},
             [&](int n) { copy_b(n); });
    copied();
    // The next step has landed: after its copies came those of AHEAD - 1 steps, and in
    // the first AHEAD - 1 steps of a tile the stores of the tile before.
    constexpr int W = (AHEAD - 1) * (NH + NB) + (EARLY ? S_ALL : 0);
    wait_vmcnt_lgkm0<(W < 63 ? W : 63)>();
    __builtin_amdgcn_s_barrier();
    ra = ra + 1 == NSLOT ? 0 : ra + 1;
    rb = ra;
    sub_step(blocks, I3{}, fa1, fb[0], next_tag, [&](int n) { read_a(fa0, 0, n); }, I1{}, I0{}, nothing);
    if constexpr (decltype(next_tag)::value) {
#pragma unroll
      for (int j = 0; j < TN; ++j) read_b(0, j);
    }
    take_scales(0);
    fence();
  };
  // bf16 by groups: step Q of one.  The group's weights are all in registers after the first
  // step, so that their slot is free for the copies of two groups on; EARLY: the first
  // AHEAD - 1 steps of a tile.
  auto group_step = [&](auto blocks, auto next_tag, auto early_tag, auto q_tag)
                        __attribute__((always_inline)) {
    constexpr bool EARLY = decltype(early_tag)::value;
    constexpr int Q = decltype(q_tag)::value, BLOCKS = decltype(blocks)::value;
    constexpr int NEXT = decltype(next_tag)::value, WEIGHTS = Q == 0 && BLOCKS ? TN : 0;
    using Reads = std::integral_constant<int, BLOCKS + WEIGHTS>;
    const u32x4_t* const w = fb[Q];
    sub_step(blocks, I0{}, fa0, w, Reads{}, [&](int n) {
      if (n < BLOCKS) read_a(fa1, 1, n);
      else read_b(1, n - BLOCKS);
    }, I1{}, I0{}, nothing);
    sub_step(blocks, I1{}, fa1, w, Reads{}, [&](int n) {
      if (n < BLOCKS) read_a(fa0, 2, n);
      else read_b(2, n - BLOCKS);
    }, I2{}, CopiesA{}, [&](int n) { copy_a(n); });
    sub_step(blocks, I2{}, fa0, w, Reads{}, [&](int n) {
      if (n < BLOCKS) read_a(fa1, 3, n);
      else read_b(3, n - BLOCKS);
    }, I1{}, std::integral_constant<int, Q == 1 || Q == 2>{}, [&](int) { copy_s(Q - 1); });
    // The next step has landed: after its activations came the weights' copy of that step
    // and the copies of AHEAD - 1 steps (this step's weights' not yet), two scales among any
    // four steps, and in the first AHEAD - 1 steps of a tile the stores of the tile before.
    // The next group's weights are older than that.
    constexpr int W = (AHEAD - 1) * (NH + 1) + 2 + (EARLY ? S_ALL : 0);
    wait_vmcnt_lgkm0<(W < 63 ? W : 63)>();
    __builtin_amdgcn_s_barrier();
    ra = ra + 1 == NSLOT ? 0 : ra + 1;
    if constexpr (Q == 3) rb ^= 1;
    constexpr int GROUP = Q == 3 && NEXT ? 3 * TN : 0;
    sub_step(blocks, I3{}, fa1, w, std::integral_constant<int, NEXT + GROUP>{}, [&](int n) {
      if (n < NEXT) read_a(fa0, 0, n);
      else if (n < NEXT + TN) read_b(0, n - NEXT);
      else read_s((n - NEXT - TN) / 2, (n - NEXT - TN) % 2);
    }, I1{}, I1{}, [&](int) { copy_b(Q); });
    copied();
    if constexpr (Q == 3) copied_b();
    if constexpr (NEXT > 0) to_numbers((Q + 1) % 4);
    fence();
  };
  using Early = std::true_type;
  using Later = std::false_type;
  // A tile's steps in a wave of which the first BLOCKS 32-row blocks have rows.  The last
  // reads are of the next tile, of all blocks.
  auto steps = [&](auto blocks) __attribute__((always_inline)) {
    if constexpr (MX4 && LDS_SCALES) {
      first_subs(blocks, Early{}, I0{}, 0);          // (nk >= 3)
      for (int kt = 1; kt < nk; ++kt) {
        if (kt == nk - 2) begin_copies(nxt, more);   // two steps before the tile's end
        last_sub(blocks, blocks);
        first_subs(blocks, Later{}, I0{}, 0);
      }
      last_sub(blocks, All{});
    } else if constexpr (MX4) {
      first_subs(blocks, Early{}, I0{}, 2);
      // step kt, its scales in one set and those of two steps on going there; the copies
      // and scales reach the next tile two steps before its end
      auto step = [&](auto set_tag, int kt) __attribute__((always_inline)) {
        if (kt == nk - 2) {
          begin_copies(nxt, more);
          begin_scales(nxt);
        }
        last_sub(blocks, blocks);
        first_subs(blocks, Later{}, set_tag, kt + 2 < nk ? kt + 2 : kt + 2 - nk);
      };
      int kt = 1;
      for (; kt + 1 < nk; kt += 2) {
        step(I1{}, kt);
        step(I0{}, kt + 1);
      }
      if (kt < nk) {
        step(I1{}, kt);
      } else {                                       // an odd number: the sets change places
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const uint32_t v = sa_next[0][i];
          sa_next[0][i] = sa_next[1][i];
          sa_next[1][i] = v;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const uint32_t v = sb_next[0][j];
          sb_next[0][j] = sb_next[1][j];
          sb_next[1][j] = v;
        }
      }
      last_sub(blocks, All{});
    } else if constexpr (GROUPED) {
      group_step(blocks, blocks, Early{}, I0{});     // (G >= 3)
      group_step(blocks, blocks, Early{}, I1{});
      group_step(blocks, blocks, Early{}, I2{});
      group_step(blocks, blocks, Later{}, I3{});
      for (int g = 1; g < G - 1; ++g) {
        if (g == G - 2) begin_b(nxt, more);          // the weights' copies reach the next tile
        group_step(blocks, blocks, Later{}, I0{});
        group_step(blocks, blocks, Later{}, I1{});
        group_step(blocks, blocks, Later{}, I2{});
        group_step(blocks, blocks, Later{}, I3{});
      }
      begin_a(nxt);                                  // and the activations'
      group_step(blocks, blocks, Later{}, I0{});
      group_step(blocks, blocks, Later{}, I1{});
      group_step(blocks, blocks, Later{}, I2{});
      group_step(blocks, All{}, Later{}, I3{});
    } else {
      int kt = 0;
      for (; kt < AHEAD - 1; ++kt) bf16_step(blocks, blocks, Early{}, kt + 1);
      for (; kt < nk - AHEAD; ++kt) bf16_step(blocks, blocks, Later{}, kt + 1);
      begin_copies(nxt, more);                       // the copies reach the next tile
      for (; kt < nk - 1; ++kt) bf16_step(blocks, blocks, Later{}, kt + 1);
      begin_scales(nxt);                             // and the scales
      bf16_step(blocks, All{}, Later{}, 0);
    }
  };
  while (true) {
    zero_acc();
    const int left = cur.rows - wm * WTM;
    if (BM == 256 || left > WTM / 2) steps(All{});
    else if (left > 0) steps(std::integral_constant<int, TM / 2>{});
    else steps(I0{});
    const BigTile done = cur;
    const bool go_on = more;
    cur = nxt;
    ++round;
    more = go_on && tile_of(round) < n_tiles;
    if (more) {                                      // rows of the tile after the next
      nxt = load_entry(tile_of(round));
      load_rows(nxt);
    }
    __builtin_amdgcn_sched_barrier(0);               // the stores come after, see the waits
#pragma unroll
    for (int i = 0; i < TM; ++i) store_block<ACT, EPI, WTM>(p, done, i, wm, wn, lane, acc[i]);
    __builtin_amdgcn_sched_barrier(0);
    if (!go_on) break;
    finish_rows(nxt, more);                          // (loaded ahead of the stores)
  }
  wait_vmcnt<0>();                                   // no copy outlives the workgroup
}

// ---------------------------------------------------------------------------
// What the products need first, in one launch: their tile lists, and the scales of
// gathered MX4 activations in routed order.
// ---------------------------------------------------------------------------
struct BigList : TileList {
  int bm;
};

// An expert's rows are spread over its tiles in equal numbers of 32-row blocks.  128-row
// tiles, whose waves leave out the blocks without rows, are listed by classes of one to
// four blocks; 256-row tiles in one class.  One thread per tile: every workgroup recomputes
// the experts' starts within their classes (E <= 256) and writes the tiles of its own range
// of each list, finding a tile's expert by binary search.
__device__ __forceinline__ void build_big_lists(int block, const int32_t* __restrict__ offsets,
                                                const int32_t* __restrict__ expert_map, int E,
                                                const BigList& la, const BigList& lb) {
  __shared__ int s_wave[kTableThreads / 64][kClasses];
  __shared__ int s_start[kClasses][kTableThreads];
  __shared__ int s_total[kClasses];
  __shared__ int s_mt[kTableThreads], s_phys[kTableThreads], s_row0[kTableThreads];
  __shared__ int s_rows[kTableThreads], s_tall[kTableThreads];
  const int e = threadIdx.x;
  int row0 = 0, rows = 0, phys = -1;
  if (e < E) {
    row0 = offsets[e];
    rows = offsets[e + 1] - row0;
    phys = expert_map ? expert_map[e] : e;
  }
  s_phys[e] = phys;
  s_row0[e] = row0;
  s_rows[e] = rows;
  for (int which = 0; which < 2; ++which) {
    const BigList& L = which == 0 ? la : lb;
    if (which == 0 || la.bm != lb.bm) {
      __syncthreads();                     // (the first list has been written)
      const int mt = phys >= 0 && rows > 0 ? (rows + L.bm - 1) / L.bm : 0;
      const int tall = mt ? ((rows + mt - 1) / mt + 31) & ~31 : 0;
      const int cls = L.bm == kClasses * 32 ? kClasses - tall / 32 : 0;
      s_mt[e] = mt;
      s_tall[e] = tall;
      // sums over the experts before, of all classes at once
      int sum[kClasses];
#pragma unroll
      for (int c = 0; c < kClasses; ++c) sum[c] = cls == c ? mt : 0;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1)
#pragma unroll
        for (int c = 0; c < kClasses; ++c) {
          const int n = __shfl_up(sum[c], off, 64);
          sum[c] += (e & 63) >= off ? n : 0;
        }
      if ((e & 63) == 63)
#pragma unroll
        for (int c = 0; c < kClasses; ++c) s_wave[e >> 6][c] = sum[c];
      __syncthreads();
#pragma unroll
      for (int c = 0; c < kClasses; ++c) {
#pragma unroll
        for (int w = 0; w < kTableThreads / 64; ++w) sum[c] += w < e >> 6 ? s_wave[w][c] : 0;
        s_start[c][e] = sum[c] - (cls == c ? mt : 0);
        if (e == kTableThreads - 1) s_total[c] = sum[c];
      }
      __syncthreads();
    }
    int begin = 0, i = block * kTableThreads + e, c = 0;
    bool found = false;
    for (int k = 0; k < kClasses; ++k) {
      const int end = begin + s_total[k] * L.n_tiles;
      if (block == 0 && e == 0) L.n_entries[kClassOffset + k] = min(begin, L.max_entries);
      if (!found && i < end) {
        found = true;
        c = k;
        i -= begin;
      }
      begin = end;
    }
    if (block == 0 && e == 0) L.n_entries[kClassOffset + kClasses] = min(begin, L.max_entries);
    const int at = block * kTableThreads + e;
    if (found && at < L.max_entries) {
      int lo = 0, hi = kTableThreads - 1;  // last expert with start <= i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_start[c][mid] * L.n_tiles <= i) lo = mid;
        else hi = mid - 1;
      }
      const int x = lo;  // experts with no tiles of the class share a start; the last has some
      int m, n;
      grouped_tile(i - s_start[c][x] * L.n_tiles, s_mt[x], L.n_tiles, L.group, m, n);
      TileEntry te;
      te.row0 = s_row0[x] + m * s_tall[x];
      te.rows = min(s_tall[x], s_rows[x] - m * s_tall[x]);
      te.expert = x;
      te.phys = s_phys[x];
      te.nt = n;
      L.table[at] = te;
    }
  }
}

struct GatherScales {
  const uint64_t* src;       // [G, T] (eight blocks' scales each)
  uint64_t* dst;             // [G, R]
  const int32_t* row_src;
  long long T, R;
  int G, slots_k;
};

__global__ __launch_bounds__(kTableThreads) void mx4_prepare_kernel(
    const int32_t* __restrict__ offsets, const int32_t* __restrict__ expert_map, int E,
    BigList la, BigList lb, int list_blocks, GatherScales g) {
  if ((int)blockIdx.x < list_blocks) {
    build_big_lists(blockIdx.x, offsets, expert_map, E, la, lb);
    return;
  }
  const long long n = (long long)(gridDim.x - list_blocks) * kTableThreads;
  const int live = offsets[E];                       // rows behind the last expert's: none
  for (long long i = (long long)(blockIdx.x - list_blocks) * kTableThreads + threadIdx.x;
       i < g.R * g.G; i += n) {
    const long long group = i / g.R, r = i - group * g.R;
    if (r < live) g.dst[i] = g.src[group * g.T + g.row_src[r] / g.slots_k];
  }
}

template <int ACT, int EPI>
hipError_t launch_big(const Mx4Params& p, int bm, hipStream_t s) {
  int dev = 0, cus = 0;
  hipError_t err = hipGetDevice(&dev);
  if (err == hipSuccess) err = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (err != hipSuccess) return err;
  // one workgroup per CU, a multiple of 8 so every XCD gets the same number
  const dim3 grid(max(8, cus / 8 * 8));
  if (bm == 256)
    hipLaunchKernelGGL((gemm_mx4_big_kernel<ACT, EPI, 256>), grid, dim3(kBigThreads), 0, s, p);
  else
    hipLaunchKernelGGL((gemm_mx4_big_kernel<ACT, EPI, 128>), grid, dim3(kBigThreads), 0, s, p);
  return hipGetLastError();
}

inline int64_t list_max(int64_t R, int E, int bm, int n_tiles) {
  return (ceil_div(R, bm) + (R < E ? R : E)) * n_tiles;
}

}  // namespace

size_t mx4_big_list_bytes(int64_t R, int E, int bm, int n_cols, bool gate_up) {
  const int64_t n = list_max(R, E, bm, ceil_div(n_cols, gate_up ? kBigBN / 2 : kBigBN));
  return align_up(table_bytes(0) + (size_t)n * sizeof(TileEntry), 256);
}

hipError_t launch_mx4_prepare(const int32_t* offsets, const int32_t* expert_map, int E, int64_t R,
                              int bm_gu, int f, void* list_gu, int bm, int n_cols, void* list,
                              const uint8_t* x_scale, uint8_t* routed_scale,
                              const int32_t* row_src, int slots_k, int64_t T, int K,
                              hipStream_t s) {
  auto list_of = [&](void* at, int rows, int n_tiles) {
    const int n = (int)list_max(R, E, rows, n_tiles);   // (BIG: under 2^30)
    const TableWs t = carve_table(at, n);
    return BigList{{n_tiles, kFwdTileGroup, n, t.n_entries, t.table}, rows};
  };
  // (of one list only, both are that list: written twice, alike)
  BigList la = {}, lb = {};
  if (list_gu) la = list_of(list_gu, bm_gu, ceil_div(f, kBigBN / 2));
  if (list) lb = list_of(list, bm, ceil_div(n_cols, kBigBN));
  if (!list_gu) la = lb;
  if (!list) lb = la;
  const int blocks =
      ceil_div(la.max_entries > lb.max_entries ? la.max_entries : lb.max_entries, kTableThreads);
  GatherScales g = {};
  int more = 0;
  if (routed_scale) {
    g = {reinterpret_cast<const uint64_t*>(x_scale), reinterpret_cast<uint64_t*>(routed_scale),
         row_src, T, R, mx4_groups(K), slots_k};
    const int64_t n = (R * g.G + kTableThreads - 1) / kTableThreads;
    more = (int)(n < 4096 ? n : 4096);
  }
  hipLaunchKernelGGL(mx4_prepare_kernel, dim3(blocks + more), dim3(kTableThreads), 0, s, offsets,
                     expert_map, E, la, lb, blocks, g);
  return hipGetLastError();
}

hipError_t launch_mx4_big(const Mx4Args& a, hipStream_t s) {
  Mx4Params p = mx4_params(a);
  const TableWs t = carve_table(a.list, 0);
  p.table = t.table;
  p.n_entries = t.n_entries;
  if (a.a_scale) {
    if (a.f) return launch_big<ACT_MX4, MX4_GU>(p, a.bm, s);
    return a.f32_out ? launch_big<ACT_MX4, MX4_STORE_F32>(p, a.bm, s)
                     : launch_big<ACT_MX4, MX4_STORE>(p, a.bm, s);
  }
  if (a.f) return launch_big<ACT_BF16, MX4_GU>(p, a.bm, s);
  return a.f32_out ? launch_big<ACT_BF16, MX4_STORE_F32>(p, a.bm, s)
                   : launch_big<ACT_BF16, MX4_STORE>(p, a.bm, s);
}

}  // namespace laep
