// Grouped products at MX4 weights for many rows: the products of gemm_mx4.hip in tiles of
// 256 x 256, one persistent workgroup of eight waves (2 x 4, each 128 x 64) a CU.
//
// The k-steps of all the tiles that a workgroup walks are one stream: copies run two
// steps (three for bf16 activations) ahead of the matrix instructions, past a tile's end
// into the next tile, whose token rows were read a tile earlier, and so do the reads of
// fragments.  A tile's epilogue, from registers to memory, lies between two steps with
// the next tile's operands landed or in flight.
//   MX4:  a step is 256 columns, 32 KB ("half") of each operand; the LDS is a ring of
//         five halves (A0 B0 A1 B1 A2 | B2 A3 ...).  Scales go straight to registers, one
//         dword per fragment and step; those of gathered activations lie in routed order
//         (a scale of a gathered row would cost a cache line a step, as much as its codes).
//   bf16: a step is 64 columns, 32 KB of activations and 8 KB of weight codes; the LDS
//         is a ring of four.
#include <type_traits>

#include "gemm_mx4.hpp"

namespace laep {
namespace {

constexpr int kBigThreads = 512;
constexpr int kBigBN = 256;

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
  constexpr int APART = BM * 128;                    // a step's activations
  constexpr int BPART = MX4 ? kBigBN * 128 : kBigBN * 32;  // and its weights
  // steps in the LDS: of A; of B (256 rows in MX4: one fewer)
  constexpr int NSLOT = MX4 ? 3 : BM == 256 ? 4 : 6;
  constexpr int NSLOTB = MX4 && BM == 256 ? 2 : NSLOT;
  constexpr int AHEAD = MX4 ? 2 : NSLOT - 1;         // steps the copies run ahead
  constexpr int NH = APART / 16 / NT;                // copies a thread and step of A
  constexpr int NB = BPART / 16 / NT;                // and of B
  static_assert(BM == 256 || BM == 128, "two rows of waves");
  constexpr int SMEM = NSLOT * APART + NSLOTB * BPART;
  static_assert(SMEM <= 160 * 1024, "the LDS");
  __shared__ __attribute__((aligned(1024))) char smem[SMEM];

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5;
  const int wm = wave / 4, wn = wave % 4;
  // this XCD's contiguous range of the tile list (block i runs on XCD i % 8), dealt to
  // its workgroups in turn
  const int n_valid = *p.n_entries;
  const int per = (n_valid + 7) >> 3, stride = gridDim.x >> 3;
  const int t_lo = (blockIdx.x & 7) * per, t_hi = min(t_lo + per, n_valid);
  int next = t_lo + (blockIdx.x >> 3);
  if (next >= t_hi) return;

  auto load_entry = [&](int at) {   // through the scalar cache
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
      const int rr = r < t.rows ? r : t.rows - 1;    // rows past the tile's end: any valid row
      raw[i] = p.row_src ? (uint32_t)p.row_src[t.row0 + rr] : (uint32_t)rr;
    }
  };
  uint32_t a_voff[NH], b_voff;
  int b_group[NB];                                   // byte offsets of 64-row groups
  __amdgpu_buffer_rsrc_t a_rsrc, b_rsrc;
  int c_step = 0;                                    // step of its tile that is copied next
  const int a_lc = (tid & 7) ^ swz8(tid >> 3);       // chunk of a row (64 rows on: the same)
  // (no tile left: the copies are dropped)
  auto begin_copies = [&](const BigTile& t, bool left) {
    const long long row0 = p.row_src ? 0 : t.row0;
#pragma unroll
    for (int i = 0; i < NH; ++i) {
      const uint32_t row = p.row_src ? raw[i] / (uint32_t)p.slots_k : raw[i];
      a_voff[i] = left ? row * (uint32_t)a_row_bytes + a_lc * 16 : kDroppedCopy;
    }
    // a 64-row group of the tile lies in the matrix or past it (f and N are multiples of
    // 64: past it, the first group again); bf16: two chunks a row, rows 4 apart swap them
    const int r = MX4 ? tid >> 3 : tid >> 1;
    const int lc = MX4 ? a_lc : (tid & 1) ^ ((r >> 2) & 1);
    if constexpr (MX4) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int at = EPI == MX4_GU ? 32 * i : 64 * i;
        const bool in = EPI == MX4_GU ? t.nt * 128 + at < p.f : t.nt * 256 + at < p.N;
        b_group[i] = in ? at * (p.K / 2) : 0;
      }
    }
    b_voff = left ? (uint32_t)weight_row(t.nt, r) * (uint32_t)(p.K / 2) + lc * 16 : kDroppedCopy;
    a_rsrc = mx4_rsrc(static_cast<const char*>(p.A) + row0 * a_row_bytes);
    b_rsrc = mx4_rsrc(p.B + (long long)t.phys * p.N * (p.K / 2));
    c_step = 0;
  };
  // MX4: the columns of the last, partial 256 that lie past K are dropped
  auto codes_at = [&](uint32_t voff) {
    return c_step * kMx4Group + a_lc * kMx4Block < p.K ? voff : kDroppedCopy;
  };
  int a_slot = 0, b_slot = 0;
  auto copy_a = [&](int i) {
    char* const dst = smem + a_slot * APART + i * NT * 16;
    const uint32_t v[1] = {MX4 ? codes_at(a_voff[i]) : a_voff[i]};
    dma_chunks<1, NT>(dst, a_rsrc, v, c_step * 128, wave);
  };
  auto copy_b = [&](int i) {
    char* const dst = smem + NSLOT * APART + b_slot * BPART + i * NT * 16;
    const uint32_t v[1] = {MX4 ? codes_at(b_voff) : b_voff};
    dma_chunks<1, NT>(dst, b_rsrc, v, MX4 ? b_group[i] + c_step * 128 : c_step * 32, wave);
  };
  auto copied = [&]() {                              // both operands of a step are issued
    ++c_step;
    a_slot = a_slot + 1 == NSLOT ? 0 : a_slot + 1;
    b_slot = b_slot + 1 == NSLOTB ? 0 : b_slot + 1;
  };

  // ---- scales of a step: a dword per fragment (MX4: two steps ahead, in two sets), or
  // the byte of the lane's block (bf16)
  constexpr int NSET = MX4 ? 2 : 1;
  uint32_t sa[TM], sb[TN], sa_next[NSET][TM], sb_next[NSET][TN], sa_off, sb_off;
  int sb_far;                                        // from fragment 0's scales to 1's
  __amdgpu_buffer_rsrc_t sa_rsrc, sb_rsrc;
  auto begin_scales = [&](const BigTile& t) {
    if constexpr (MX4) {
      // rows past the tile's end take other rows' scales, past the array's end none
      sa_off = (wm * WTM + (lane & 31)) * 8 + half * 4;
      sa_rsrc = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(p.a_scale) + (long long)t.row0 * 8, 0,
          (int)((G * p.a_rows - t.row0) * 8), kBufferFlags);
    }
    // fragment 1: the up rows, or the odd columns
    sb_off = weight_row(t.nt, wn * 64 + (lane & 31)) * 8 + half * (MX4 ? 4 : 1);
    sb_far = EPI == MX4_GU ? p.f * 8 : 8;
    sb_rsrc = mx4_rsrc(p.b_scale + (long long)t.phys * G * p.N * 8);
  };
  constexpr int NS = MX4 ? TM + TN : TN;
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
    b_off[j] = MX4 ? r * 128 + (((4 * half) ^ swz8(r)) << 4)
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
  u32x4_t fb[MX4 ? 4 : 1][TN];                       // MX4: a step's B whole; bf16: its codes
  int ra = 0, rb = 0;                                // slots that are read
  auto a_base = [&]() { return smem + ra * APART; };
  auto b_base = [&]() { return smem + NSLOT * APART + rb * BPART; };
  auto read_a = [&](u32x4_t* ga, int s, int i) {
    ga[i] = *reinterpret_cast<const u32x4_t*>(a_base() + (a_off[i & 1] ^ (s << 4)) + (i >> 1) * 8192);
  };
  auto read_b = [&](int s, int j) {
    fb[s][j] = *reinterpret_cast<const u32x4_t*>(b_base() + (b_off[j] ^ (s << 4)));
  };
  // Sub-step S on fa, beside its matrix instructions READS fragment reads (of what later
  // sub-steps take), and extra(n) at every EVERY-th of them, COUNT times.
  auto sub_step = [&](auto s_tag, const u32x4_t* fa, auto reads_tag, auto read, auto every_tag,
                      auto count_tag, auto extra) {
    constexpr int S = decltype(s_tag)::value, EVERY = decltype(every_tag)::value;
    constexpr int COUNT = decltype(count_tag)::value, READS = decltype(reads_tag)::value;
    constexpr int NMM = TM * TN, SLOTS = EVERY * COUNT;
    constexpr int WORK = NMM > READS ? NMM : READS, MOST = WORK > SLOTS ? WORK : SLOTS;
    u32x4_t wv[TN];
    if constexpr (!MX4) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
        wv[j] = mx4_values8_bf16(fb[0][j][S], __uint_as_float(sb[j]));
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
  using ReadsA = std::integral_constant<int, TM>;
  using Scales = std::integral_constant<int, NS>;
  auto nothing = [](int) {};

  // ---- the stream
  BigTile cur = load_entry(next), nxt = cur;
  load_rows(cur);
  begin_copies(cur, true);
  begin_scales(cur);
#pragma unroll
  for (int t = 0; t < AHEAD; ++t) {
#pragma unroll
    for (int i = 0; i < NH; ++i) copy_a(i);
#pragma unroll
    for (int i = 0; i < NB; ++i) copy_b(i);
    copied();
  }
  if constexpr (MX4) {                               // (A runs one step further ahead)
#pragma unroll
    for (int i = 0; i < NH; ++i) copy_a(i);
  }
#pragma unroll
  for (int t = 0; t < NSET; ++t)
#pragma unroll
    for (int n = 0; n < NS; ++n) load_scale(t, n, t);
  next += stride;
  bool more = next < t_hi;
  if (more) {
    nxt = load_entry(next);
    load_rows(nxt);
  }
  wait_vmcnt<0>();                                   // (once a workgroup)
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < TM; ++i) read_a(fa0, 0, i);
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int s = 0; s < (MX4 ? 3 : 1); ++s) read_b(s, j);
  if constexpr (!MX4) take_scales(0);
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
  // of the next step's first fragments, and the copies of A two steps past that one into
  // the slot that the step has just freed.
  auto last_sub = [&]() {
    sub_step(I3{}, fa1, std::integral_constant<int, TM + 3 * TN>{}, [&](int n) {
      if (n < TN) read_b(0, n);
      else if (n < TN + TM) read_a(fa0, 0, n - TN);
      else read_b(1 + (n - TN - TM) / TN, (n - TN - TM) % TN);
    }, I1{}, CopiesA{}, [&](int n) { copy_a(n); });
    fence();
  };
  // MX4: the rest of a step.  Its B fragments are all in registers after the first
  // sub-step, so that B's slot is free for the copies of two steps on.
  auto first_subs = [&](auto early_tag, auto set_tag, int s_step) {
    constexpr bool EARLY = decltype(early_tag)::value;
    constexpr int SET = decltype(set_tag)::value;
    take_scales(SET);
    sub_step(I0{}, fa0, std::integral_constant<int, TM + TN>{}, [&](int n) {
      if (n < TM) read_a(fa1, 1, n);
      else read_b(3, n - TM);
    }, I1{}, Scales{}, [&](int n) { load_scale(SET, n, s_step); });
    if constexpr (NSLOTB == 2) {                     // (with three slots B's is free already)
      wait_lgkm0();
      __builtin_amdgcn_s_barrier();
    }
    sub_step(I1{}, fa1, ReadsA{}, [&](int n) { read_a(fa0, 2, n); },
             std::integral_constant<int, TM / 2>{}, CopiesB{}, [&](int n) { copy_b(n); });
    copied();
    sub_step(I2{}, fa0, ReadsA{}, [&](int n) { read_a(fa1, 3, n); }, I1{}, I0{}, nothing);
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
  auto bf16_step = [&](auto early_tag, int s_step) {
    constexpr bool EARLY = decltype(early_tag)::value;
    sub_step(I0{}, fa0, ReadsA{}, [&](int n) { read_a(fa1, 1, n); }, I1{}, Scales{},
             [&](int n) { load_scale(0, n, s_step); });
    sub_step(I1{}, fa1, ReadsA{}, [&](int n) { read_a(fa0, 2, n); }, I2{}, CopiesA{},
             [&](int n) { copy_a(n); });
    sub_step(I2{}, fa0, ReadsA{}, [&](int n) { read_a(fa1, 3, n); }, I1{}, CopiesB{},
             [&](int n) { copy_b(n); });
    copied();
    // The next step has landed: after its copies came those of AHEAD - 1 steps, and in
    // the first AHEAD - 1 steps of a tile the stores of the tile before.
    constexpr int W = (AHEAD - 1) * (NH + NB) + (EARLY ? S_ALL : 0);
    wait_vmcnt_lgkm0<(W < 63 ? W : 63)>();
    __builtin_amdgcn_s_barrier();
    ra = ra + 1 == NSLOT ? 0 : ra + 1;
    rb = ra;
    sub_step(I3{}, fa1, ReadsA{}, [&](int n) { read_a(fa0, 0, n); }, I1{}, I0{}, nothing);
#pragma unroll
    for (int j = 0; j < TN; ++j) read_b(0, j);
    take_scales(0);
    fence();
  };
  using Early = std::true_type;
  using Later = std::false_type;
  while (true) {
    zero_acc();
    if constexpr (MX4) {
      first_subs(Early{}, I0{}, 2);                  // (nk >= 3)
      // step kt, its scales in one set and those of two steps on going there; the copies
      // and scales reach the next tile two steps before its end
      auto step = [&](auto set_tag, int kt) {
        if (kt == nk - 2) {
          begin_copies(nxt, more);
          begin_scales(nxt);
        }
        last_sub();
        first_subs(Later{}, set_tag, kt + 2 < nk ? kt + 2 : kt + 2 - nk);
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
      last_sub();
    } else {
      int kt = 0;
      for (; kt < AHEAD - 1; ++kt) bf16_step(Early{}, kt + 1);
      for (; kt < nk - AHEAD; ++kt) bf16_step(Later{}, kt + 1);
      begin_copies(nxt, more);                       // the copies reach the next tile
      for (; kt < nk - 1; ++kt) bf16_step(Later{}, kt + 1);
      begin_scales(nxt);                             // and the scales
      bf16_step(Later{}, 0);
    }
    const BigTile done = cur;
    const bool go_on = more;
    cur = nxt;
    next += stride;
    more = go_on && next < t_hi;
    if (more) {                                      // rows of the tile after the next
      nxt = load_entry(next);
      load_rows(nxt);
    }
    __builtin_amdgcn_sched_barrier(0);               // the stores come after, see the waits
#pragma unroll
    for (int i = 0; i < TM; ++i) store_block<ACT, EPI, WTM>(p, done, i, wm, wn, lane, acc[i]);
    __builtin_amdgcn_sched_barrier(0);
    if (!go_on) break;
  }
  wait_vmcnt<0>();                                   // no copy outlives the workgroup
}

// ---------------------------------------------------------------------------
// What the products need first, in one launch: their tile lists, and the scales of
// gathered MX4 activations in routed order.
// ---------------------------------------------------------------------------
struct GatherScales {
  const uint64_t* src;       // [G, T] (eight blocks' scales each)
  uint64_t* dst;             // [G, R]
  const int32_t* row_src;
  long long T, R;
  int G, slots_k;
};

__global__ __launch_bounds__(kTableThreads) void mx4_prepare_kernel(
    const int32_t* __restrict__ offsets, const int32_t* __restrict__ expert_map, int E,
    int BM, TileList la, TileList lb, int list_blocks, GatherScales g) {
  if ((int)blockIdx.x < list_blocks) {
    build_tile_lists(blockIdx.x, offsets, expert_map, E, BM, la, lb);
    return;
  }
  const long long n = (long long)(gridDim.x - list_blocks) * kTableThreads;
  const int live = offsets[E];                       // rows behind the last expert's: none
  for (long long r = (long long)(blockIdx.x - list_blocks) * kTableThreads + threadIdx.x;
       r < g.R && r < live; r += n) {
    const long long t = g.row_src[r] / g.slots_k;
    for (int i = 0; i < g.G; ++i) g.dst[i * g.R + r] = g.src[i * g.T + t];
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

inline int list_max(int64_t R, int E, int bm, int n_tiles) {
  return (ceil_div(R, bm) + (int)(R < E ? R : E)) * n_tiles;
}

}  // namespace

size_t mx4_big_list_bytes(int64_t R, int E, int bm, int n_cols, bool gate_up) {
  return table_bytes(list_max(R, E, bm, ceil_div(n_cols, gate_up ? kBigBN / 2 : kBigBN)));
}

hipError_t launch_mx4_prepare(const int32_t* offsets, const int32_t* expert_map, int E, int64_t R,
                              int bm, int f, void* list_gu, int n_cols, void* list,
                              const uint8_t* x_scale, uint8_t* routed_scale,
                              const int32_t* row_src, int slots_k, int64_t T, int K,
                              hipStream_t s) {
  const int nt_a = list_gu ? ceil_div(f, kBigBN / 2) : 1, nt_b = ceil_div(n_cols, kBigBN);
  const int max_a = list_gu ? list_max(R, E, bm, nt_a) : 0, max_b = list_max(R, E, bm, nt_b);
  const TableWs tb = carve_table(list, max_b);
  const TableWs ta = list_gu ? carve_table(list_gu, max_a) : tb;
  const TileList la = {nt_a, kFwdTileGroup, max_a, ta.n_entries, ta.table};
  const TileList lb = {nt_b, kFwdTileGroup, max_b, tb.n_entries, tb.table};
  const int blocks = ceil_div(max_a > max_b ? max_a : max_b, kTableThreads);
  GatherScales g = {};
  int more = 0;
  if (routed_scale) {
    g = {reinterpret_cast<const uint64_t*>(x_scale), reinterpret_cast<uint64_t*>(routed_scale),
         row_src, T, R, mx4_groups(K), slots_k};
    more = (int)(ceil_div(R, kTableThreads) < 4096 ? ceil_div(R, kTableThreads) : 4096);
  }
  // (of one list only, both are that list: written twice, alike)
  hipLaunchKernelGGL(mx4_prepare_kernel, dim3(blocks + more), dim3(kTableThreads), 0, s, offsets,
                     expert_map, E, bm, list_gu ? la : lb, lb, blocks, g);
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
