// Balance loss of the router (moe_balance_loss, moe_balance_loss_bwd).  With p the
// softmax of the alive experts' logits and the T tokens cut into sequences s of
// n_s tokens,
//   counts[s, e] = slots of s routed to e,  P[s, e] = mean over s of p[t, e],
//   f[s, e] = N_alive counts[s, e] / (k n_s),
//   loss = coef * mean over the non-empty s of sum_e f[s, e] P[s, e],
//   c[s, e] = coef f[s, e] / (n_s S_nonempty)     (= dloss / dp[t, e]),
//   dlogits[t, e] = dloss p_e (c_e - sum_i p_i c_i).
// HBM-bound where long, launch-bound where short.
//
// The tokens are cut into equal chunks, one workgroup each, whatever the sequences:
// walking chunks and sequences in token order, each step goes to the next chunk or to
// the next sequence, so the pair (chunk c, sequence s) has the slot c + s to itself,
// and the partial sums need n_chunks + n_seq slots however the sequences fall.  A
// second pass sums each sequence's slots in order.  Counts are integers; every
// floating-point sum has a fixed order.
//
// A token's row belongs to G lanes of four experts each (G the power of two from
// E / 4 up), so a wave reads 64 / G rows at a time in whole lines and a softmax takes
// log2 G lane moves for its maximum and its sum.  The vector units are as busy as HBM
// where G lanes hold far fewer than 4 G experts (68 instructions a row and wave in the
// first pass), so row addresses are a scalar base and the lane's own place, and rows inside
// a segment are not checked: 83022 tokens of 77 experts in 25 sequences, forward and
// backward, 30.9 us for 36.6, 32768 of 45 in 24 18.2 for 20.7.
#include <type_traits>

#include "common.hpp"
#include "internal.hpp"
#include "lanes.hpp"

namespace laep {
namespace {

constexpr int kBalThreads = 256;
constexpr int kBalWaves = kBalThreads / kWave;
constexpr int kBalMaxE = 256;
constexpr int kBalAhead = 4;         // rows of a lane group in flight
constexpr int kBalIds = 4;           // slots of a thread loaded ahead
constexpr int kBalMaxChunks = 1024;
constexpr int kSumThreads = 1024, kSumCols = 64, kSumColsFew = 16;   // second pass
constexpr int kLastParts = 32;       // parts of the loss that the last workgroup adds

struct BalWs {          // carved from the workspace
  int* live;            // non-empty sequences
  int* done;            // workgroups of the second pass that have their part of the loss
  float* part_p;        // [slots, Ep], Ep: E rounded up to 4
  int* part_n;          // [slots, Ep]
  float* part_loss;     // [n_seq, column blocks], or kLastParts
};

__host__ __device__ inline int bal_ep(int E) { return (E + 3) & ~3; }
inline int bal_lanes(int E) {
  int g = 1;
  while (4 * g < E) g *= 2;
  return g;
}
inline int bal_blocks(int E, int cols) { return (E + cols - 1) / cols; }

// Tokens per chunk: two passes of the workgroup's rows at least, and 32; fewer where that
// would put many sequences into a chunk, which takes them one after the other (about
// 0.7 us each: 60 sequences of 500 tokens in all over 2 experts, trained, 21 us, in one
// chunk 45; with two tokens at least 900 sequences of 1000 tokens take 20 us, with eight 31).
constexpr int kBalLeast = 2;
inline int bal_cut(int tokens, int T, int n_seq) {   // to about two sequences
  const int two = 2 * (T / n_seq);
  if (n_seq == 1 || two >= tokens) return tokens;
  return two > kBalLeast ? two : kBalLeast;
}
inline int bal_chunk(int T, int E, int n_seq) {
  const int rows = 2 * kBalThreads / bal_lanes(E);
  const int least = bal_cut(rows > 32 ? rows : 32, T, n_seq);
  const int few = T > 0 ? (T - 1) / kBalMaxChunks + 1 : 1;
  return few > least ? few : least;
}
inline int bal_chunks(int T, int chunk) { return T > 0 ? (T - 1) / chunk + 1 : 1; }

// A workspace for the largest call serves the smaller ones: the number of chunks falls
// where a chunk gains a token, E a lane or n_seq a sequence, so the space is for what
// never falls.
inline size_t bal_carve(void* ws, int T, int E, int S, BalWs& w) {
  char* p = static_cast<char*>(ws);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* const r = p + at;
    at += align_up(bytes, 256);
    return r;
  };
  const int most = T > 0 ? (T - 1) / kBalLeast + 1 : 1;
  const size_t cells = ((size_t)(most < kBalMaxChunks ? most : kBalMaxChunks) + S) * bal_ep(E);
  w.live = reinterpret_cast<int*>(take(8));
  w.done = w.live + 1;
  w.part_p = reinterpret_cast<float*>(take(cells * 4));
  w.part_n = reinterpret_cast<int*>(take(cells * 4));
  const size_t parts = (size_t)S * bal_blocks(E, kSumCols);
  w.part_loss = reinterpret_cast<float*>(take((parts > kLastParts ? parts : kLastParts) * 4));
  return at;
}

// Token range of sequence s (no offsets: one sequence of all tokens), inside [0, T].
__device__ __forceinline__ void seq_range(const int32_t* __restrict__ off, int s, int T, int& a,
                                          int& b) {
  a = off ? min(max(off[s], 0), T) : 0;
  b = off ? min(max(off[s + 1], a), T) : T;
}

// First sequence that ends after token t (n_seq if none does), by the whole wave: 64
// ends are compared at a time, so 64 sequences take one load and not a chain of six.
__device__ __forceinline__ int first_seq(const int32_t* __restrict__ off, int n_seq, int t) {
  if (!off) return 0;
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, len = n_seq;   // the answer lies in [lo, lo + len]
  while (len > 0) {
    const int piece = (len + kWave - 1) / kWave;
    const bool past = lane * piece < len && off[lo + min((lane + 1) * piece, len)] <= t;
    const int n = min((int)__popcll(__ballot(past)) * piece, len);   // ended by t
    lo += n;
    len = piece == 1 ? 0 : min(piece - 1, len - n);
  }
  return lo;
}

// The sequence to go on with after one that is empty at token t: the next that ends past
// t, for the loop's own step to reach (forwards whatever the offsets hold).  t is the
// empty one's own place, not the last token done: tokens of no sequence may lie between.
// 2000 sequences of 4 tokens in all: 21 us, one after the other 111.
__device__ __forceinline__ int past_empty(const int32_t* __restrict__ off, int n_seq, int s,
                                          int t) {
  return max(s, first_seq(off, n_seq, t) - 1);
}

// The four experts of a lane: e .. e + 3 of a row, whose own (alive) ones are ok.  The
// last lane of a row takes the row's last four where E is no multiple of four, those of
// the lane before being not its own; lanes past the row own none.  With fewer experts
// than four, the one lane's first E.
struct Quad {
  int e;
  bool ok[4];
  bool whole;   // all four of the row, whatever is alive
};
__device__ __forceinline__ Quad quad_of(int lane, int E, const uint8_t* __restrict__ alive) {
  Quad q;
  const int e0 = 4 * lane;
  q.e = max(0, min(e0, E - 4));
  uint8_t a[4];   // (loaded together, whatever is masked)
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = alive == nullptr ? 1 : alive[min(q.e + i, E - 1)];
#pragma unroll
  for (int i = 0; i < 4; ++i) q.ok[i] = q.e + i >= e0 && q.e + i < E && a[i] != 0;
  q.whole = e0 + 4 <= E;
  return q;
}
// expert i of a lane is its own, alive or not
__device__ __forceinline__ bool own(const Quad& q, int lane, int i, int E) {
  return q.e + i >= 4 * lane && q.e + i < E;
}

// Streaming loads of a lane's four: what the caches hold is still found there, and the
// rest does not push out what other calls wrote (131072 x 256, first pass: 43 -> 28 us).
// VEC: E is a multiple of four and rows are 16-byte aligned; else the four are loaded
// together all the same, 4-byte aligned (131072 tokens trained, four single loads / one:
// 250 experts 92 / 84 us, 131 62 / 58, though 45 25.4 / 26.3).
typedef f32x4_t f32x4_a4_t __attribute__((aligned(4)));
template <bool VEC>
__device__ __forceinline__ f32x4_t load4(const float* __restrict__ p, int E) {
  if constexpr (VEC) return ld_stream(reinterpret_cast<const f32x4_t*>(p));
  if (E >= 4) return __builtin_nontemporal_load(reinterpret_cast<const f32x4_a4_t*>(p));
  return f32x4_t{p[0], E > 1 ? p[1] : 0.0f, E > 2 ? p[2] : 0.0f, 0.0f};
}

// exp(l - m) of a row over its G lanes, m its maximum; returns 1 / their sum.  exp(l - m)
// is taken as 2^((l - m) log2 e): one subtraction, one product and the hardware's exp2 (an
// ulp) instead of a library call of a dozen instructions.  The maximum is subtracted first:
// it then gives exactly 1 whatever its size, rows of one finite mask value are uniform, and
// no finite logit overflows (a difference past the range is -inf, hence 0).  A row without a
// logit above -inf gets zeros.
template <int G>
__device__ __forceinline__ float exps4(const bool ok[4], const f32x4_t& l, float v[4]) {
  constexpr float kLog2e = 1.44269504f;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = ok[i] ? l[i] : -INFINITY;
    m = fmaxf(m, v[i]);
  }
  m = lanes_max<G>(m);
  const float base = m == -INFINITY ? 0.0f : m;
  float z = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = __builtin_amdgcn_exp2f((v[i] - base) * kLog2e);
    z += v[i];
  }
  z = lanes_sum<G>(z);
  return z == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(z);   // else z >= 1 (or a NaN)
}

// f(row, the lane's four logits, row < n) for the rows of a segment of n, kBalAhead loads
// in flight.  The addresses are a uniform base and the lane's place; rows past the segment
// load its last row's bytes.
template <bool VEC, int ROWS, typename F>
__device__ __forceinline__ void walk_rows(const float* seg, int n, int E, int first, int e, F f) {
  const unsigned at = first * E + e;
  int r = 0;
  for (; r + ROWS * kBalAhead <= n; r += ROWS * kBalAhead) {  // (uniform)
    f32x4_t l[kBalAhead];
#pragma unroll
    for (int u = 0; u < kBalAhead; ++u) l[u] = load4<VEC>(seg + (size_t)(r + u * ROWS) * E + at, E);
#pragma unroll
    for (int u = 0; u < kBalAhead; ++u) f(r + u * ROWS + first, l[u], true);
  }
  if (r >= n) return;
  f32x4_t l[kBalAhead];
#pragma unroll
  for (int u = 0; u < kBalAhead; ++u)
    l[u] = load4<VEC>(seg + (size_t)min(r + u * ROWS + first, n - 1) * E + e, E);
#pragma unroll
  for (int u = 0; u < kBalAhead; ++u)
    if (r + u * ROWS < n) f(r + u * ROWS + first, l[u], r + u * ROWS + first < n);
}

struct BalOut {
  float* loss;
  int32_t* counts;
  float* prob_mean;
  float* grad_coef;
  float coef;
};

// One expert's outputs of a sequence of len tokens from its sums; returns its share of
// the loss.
__device__ __forceinline__ float balance_cell(const BalOut& o, size_t at, float p, int n, int len,
                                              int k, int n_alive, int live) {
  float mean = 0.0f, c = 0.0f, part = 0.0f;
  if (len > 0) {
    mean = p / (float)len;
    const float f = (float)n_alive * (float)n / ((float)k * (float)len);
    part = o.coef * f * mean / (float)live;
    c = o.coef * f / ((float)len * (float)live);
  }
  o.counts[at] = n;
  o.prob_mean[at] = mean;
  o.grad_coef[at] = c;
  return part;
}

// First pass: chunk c's probability sums and counts of each sequence in it.  ONE: the
// batch is one chunk, whose workgroup writes the results itself.
template <int G, bool VEC, bool ONE>
__global__ __launch_bounds__(kBalThreads) void balance_chunk_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ topk_idx,
    const uint8_t* __restrict__ alive, const int32_t* __restrict__ off, int T, int E, int k,
    int n_seq, int chunk, BalWs w, BalOut o) {
  constexpr int RPW = kWave / G, ROWS = kBalWaves * RPW;   // rows of a wave, of the workgroup
  __shared__ __attribute__((aligned(16))) float s_p[kBalWaves][kBalMaxE];
  __shared__ int s_n[kBalMaxE];
  __shared__ int s_live;
  __shared__ float s_loss[kBalWaves];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
  const int ep = bal_ep(E);
  int n_alive = E;
  if (ONE || blockIdx.x == gridDim.x - 1) {  // needed once: by the last workgroup, or the one
    if (tid == 0) s_live = 0;
    __syncthreads();
    int n = 0;
    for (int s = tid; s < n_seq; s += kBalThreads) {
      int a, b;
      seq_range(off, s, T, a, b);
      n += b > a;
    }
    if (n) atomicAdd(&s_live, n);
    if (ONE && alive) n_alive = __syncthreads_count(tid < E && alive[tid] != 0);
    else __syncthreads();
    if (!ONE) {
      if (tid == 0) {
        *w.live = s_live;
        *w.done = 0;
      }
      return;
    }
  }
  const Quad q = quad_of(lane % G, E, alive);
  const int t0 = blockIdx.x * chunk, t1 = T - t0 < chunk ? T : t0 + chunk;
  float loss = 0.0f;
  for (int s = ONE ? 0 : first_seq(off, n_seq, t0); s < n_seq; ++s) {
    int a, b;
    seq_range(off, s, T, a, b);
    if (!ONE && a >= t1) break;
    a = max(a, t0);
    b = min(b, t1);
    if (!ONE && a >= b) {  // (uniform)
      s = past_empty(off, n_seq, s, a);
      continue;
    }
    for (int e = tid; e < E; e += kBalThreads) s_n[e] = 0;
    __syncthreads();
    // the slots' ids: the first ones travel under the logits
    const size_t i0 = (size_t)a * k + tid, i1 = (size_t)b * k;
    int ids[kBalIds];
#pragma unroll
    for (int u = 0; u < kBalIds; ++u)
      ids[u] = i0 + u * kBalThreads < i1 ? topk_idx[i0 + u * kBalThreads] : -1;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int first = wave * RPW + lane / G;
    const auto add = [&](int, const f32x4_t& l, bool on) {
      float v[4];
      const float inv = exps4<G>(q.ok, l, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = on ? fmaf(v[i], inv, sum[i]) : sum[i];
    };
    walk_rows<VEC, ROWS>(logits + (size_t)a * E, b - a, E, first, q.e, add);
#pragma unroll
    for (int u = 0; u < kBalIds; ++u)
      if (ids[u] >= 0 && ids[u] < E) atomicAdd(&s_n[ids[u]], 1);
    for (size_t i = i0 + kBalIds * kBalThreads; i < i1; i += kBalThreads) {
      const int e = topk_idx[i];
      if (e >= 0 && e < E) atomicAdd(&s_n[e], 1);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int d = G; d < kWave; d *= 2) sum[i] += __shfl_xor(sum[i], d, kWave);
    if (lane < G) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (own(q, lane, i, E)) s_p[wave][q.e + i] = sum[i];
    }
    __syncthreads();
    if (tid < E) {
      float p = 0.0f;
#pragma unroll
      for (int i = 0; i < kBalWaves; ++i) p += s_p[i][tid];
      if constexpr (ONE) {
        loss += balance_cell(o, (size_t)s * E + tid, p, s_n[tid], b - a, k, n_alive, s_live);
      } else {
        const size_t at = ((size_t)blockIdx.x + s) * ep + tid;
        w.part_p[at] = p;
        w.part_n[at] = s_n[tid];
      }
    }
    __syncthreads();
  }
  if constexpr (ONE) {
    loss = lanes_sum<kWave>(loss);
    if (lane == 0) s_loss[wave] = loss;
    __syncthreads();
    if (tid == 0) {
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < kBalWaves; ++i) v += s_loss[i];
      *o.loss = v;
    }
  }
}

// Second pass: COLS experts of one sequence per workgroup, its slots side by side, then
// those of a wave and of the waves in order.  16 experts a workgroup instead of 64 where
// that makes no more than kLastParts of them, for few sequences have many slots each:
// 28300 tokens of 256 experts in one sequence, forward and backward, 28.7 us for 30.5,
// 20000 of 128 17.8 for 18.7.
// The loss: alone, the workgroup has it; up to kLastParts workgroups the one that finishes
// last adds their parts, in their order (its counter was cleared by the first pass); with
// more, each of which releases the counter, a third kernel does.  Whole call, third kernel /
// last workgroup, 20000 tokens of 128 experts: 8 workgroups 13.7 / 11.6 us, 32 13.9 / 12.7,
// 64 14.1 / 13.1, 96 14.1 / 14.0, 128 14.4 / 15.0, 256 14.8 / 18.2: the two cross near 96,
// and from 32 to there the rule leaves up to a microsecond.
template <int COLS>
__global__ __launch_bounds__(kSumThreads) void balance_sum_kernel(
    const uint8_t* __restrict__ alive, const int32_t* __restrict__ off, int T, int E, int k,
    int n_seq, int chunk, BalWs w, BalOut o) {
  constexpr int LC = COLS / 4, ROWS = kSumThreads / LC, WAVES = kSumThreads / kWave;
  __shared__ __attribute__((aligned(16))) float s_p[WAVES][COLS];
  __shared__ __attribute__((aligned(16))) int s_n[WAVES][COLS];
  typedef int i32x4_t __attribute__((ext_vector_type(4)));
  const int tid = threadIdx.x, col = (tid % LC) * 4, row = tid / LC;
  const int s = blockIdx.x, e = blockIdx.y * COLS + col, ep = bal_ep(E);
  const int n_alive = alive == nullptr ? E : __syncthreads_count(tid < E && alive[tid] != 0);
  int a, b;
  seq_range(off, s, T, a, b);
  f32x4_t p = {0.f, 0.f, 0.f, 0.f};
  i32x4_t n = {0, 0, 0, 0};
  const int c0 = a / chunk, c1 = b > a ? (b - 1) / chunk : -1;
  if (c0 + tid / kWave * (kWave / LC) <= c1) {   // the wave has slots
    for (int c = c0 + row; c <= c1 && e < E; c += ROWS) {
      const size_t at = ((size_t)c + s) * ep + e;
      p += *reinterpret_cast<const f32x4_t*>(w.part_p + at);
      n += *reinterpret_cast<const i32x4_t*>(w.part_n + at);
    }
#pragma unroll
    for (int d = LC; d < kWave; d *= 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] += __shfl_xor(p[i], d, kWave);
        n[i] += __shfl_xor(n[i], d, kWave);
      }
    }
  }
  if (tid % kWave < LC) {
    *reinterpret_cast<f32x4_t*>(&s_p[tid / kWave][col]) = p;
    *reinterpret_cast<i32x4_t*>(&s_n[tid / kWave][col]) = n;
  }
  __syncthreads();
  if (tid >= kWave) return;   // one wave from here, an expert a lane
  const int my = blockIdx.y * COLS + tid;
  float part = 0.0f;
  if (tid < COLS && my < E) {
    float ps = 0.0f;
    int ns = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      ps += s_p[i][tid];
      ns += s_n[i][tid];
    }
    part = balance_cell(o, (size_t)s * E + my, ps, ns, b - a, k, n_alive, *w.live);
  }
  part = lanes_sum<kWave>(part);
  const int parts = gridDim.x * gridDim.y, mine = s * gridDim.y + blockIdx.y;
  if (parts == 1) {
    if (tid == 0) *o.loss = part;
    return;
  }
  if (parts > kLastParts) {
    if (tid == 0) w.part_loss[mine] = part;
    return;
  }
  int before = 0;
  if (tid == 0) {
    __hip_atomic_store(w.part_loss + mine, part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    before = __hip_atomic_fetch_add(w.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (__builtin_amdgcn_readfirstlane(before) != parts - 1) return;
  float v = 0.0f;
  for (int i = tid; i < parts; i += kWave)
    v += __hip_atomic_load(w.part_loss + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  v = lanes_sum<kWave>(v);
  if (tid == 0) *o.loss = v;
}

// The loss's parts, in a fixed order: one wave.
__global__ __launch_bounds__(kWave) void balance_loss_kernel(const float* __restrict__ part, int n,
                                                             float* __restrict__ loss) {
  float v = 0.0f;
  for (int i = threadIdx.x; i < n; i += 4 * kWave) {
    float p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = n - i > u * kWave ? part[i + u * kWave] : 0.0f;
    v += (p[0] + p[1]) + (p[2] + p[3]);
  }
  v = lanes_sum<kWave>(v);
  if (threadIdx.x == 0) *loss = v;
}

// Backward: a range of tokens per workgroup, walked by sequence with its coefficients
// in registers; tokens of no sequence get a zero gradient.
template <int G, bool VEC>
__global__ __launch_bounds__(kBalThreads) void balance_bwd_kernel(
    const float* logits, const float* __restrict__ grad_coef, const uint8_t* __restrict__ alive,
    const int32_t* __restrict__ off, const float* __restrict__ dloss, int T, int E, int n_seq,
    int range, float* dlogits, int accumulate) {
  constexpr int RPW = kWave / G, ROWS = kBalWaves * RPW;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
  const int l0 = lane % G, first = wave * RPW + lane / G;
  const Quad q = quad_of(l0, E, alive);
  const float scale = dloss ? *dloss : 1.0f;
  const int t0 = blockIdx.x * range, t1 = T - t0 < range ? T : t0 + range;
  auto put = [&](int t, const float v[4]) {
    float* const d = dlogits + (size_t)t * E + q.e;
    if (q.whole) {
      using V = std::conditional_t<VEC, f32x4_t, f32x4_a4_t>;
      f32x4_t r = {v[0], v[1], v[2], v[3]};
      if (accumulate) r += *reinterpret_cast<V*>(d);
      *reinterpret_cast<V*>(d) = r;
    } else if (!VEC) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (own(q, l0, i, E)) d[i] = accumulate ? d[i] + v[i] : v[i];
    }
  };
  auto zeros = [&](int from, int to) {
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!accumulate)   // (T may come near 2^31: counted from the range's start)
      for (int r = first; r < to - from; r += ROWS) put(from + r, z);
  };
  int done = t0;
  for (int s = first_seq(off, n_seq, t0); s < n_seq; ++s) {
    int a, b;
    seq_range(off, s, T, a, b);
    if (a >= t1) break;
    a = max(a, done);
    b = min(b, t1);
    if (a >= b) {  // (uniform)
      s = past_empty(off, n_seq, s, a);
      continue;
    }
    zeros(done, a);
    done = b;
    float c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = q.ok[i] ? grad_coef[(size_t)s * E + q.e + i] : 0.0f;
    const auto grad = [&](int row, const f32x4_t& l, bool on) {
      float v[4], dot = 0.0f;
      const float inv = exps4<G>(q.ok, l, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) dot += v[i] * c[i];
      dot = lanes_sum<G>(dot) * inv;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = q.ok[i] ? scale * inv * v[i] * (c[i] - dot) : 0.0f;
      if (on) put(a + row, v);
    };
    walk_rows<VEC, ROWS>(logits + (size_t)a * E, b - a, E, first, q.e, grad);
  }
  zeros(done, t1);
}

// f(lanes per row, whole vectors) for E experts
template <typename F>
void bal_shape(int E, F f) {
  auto with = [&](auto g) {
    if (E % 4 == 0) f(g, std::true_type{});
    else f(g, std::false_type{});
  };
  switch (bal_lanes(E)) {
    case 1: return with(std::integral_constant<int, 1>{});
    case 2: return with(std::integral_constant<int, 2>{});
    case 4: return with(std::integral_constant<int, 4>{});
    case 8: return with(std::integral_constant<int, 8>{});
    case 16: return with(std::integral_constant<int, 16>{});
    case 32: return with(std::integral_constant<int, 32>{});
    default: return with(std::integral_constant<int, 64>{});
  }
}

}  // namespace

size_t balance_ws_bytes(int T, int E, int n_seq) {
  BalWs w;
  return bal_carve(nullptr, T, E, n_seq, w);
}

hipError_t launch_balance(const float* logits, const int32_t* topk_idx, const uint8_t* alive,
                          const int32_t* seq_offsets, int T, int E, int k, int n_seq, float coef,
                          float* loss, int32_t* counts, float* prob_mean, float* grad_coef,
                          void* ws, hipStream_t s) {
  BalWs w;
  bal_carve(ws, T, E, n_seq, w);
  const BalOut o = {loss, counts, prob_mean, grad_coef, coef};
  // 32 passes of a workgroup's rows take no longer than two launches: 256 tokens of 64
  // experts 7.0 us for 9.4, 128 of 256 7.6 for 9.4
  const bool one = n_seq <= 4 && T <= 32 * (kBalThreads / bal_lanes(E));
  const int chunk = one ? (T > 0 ? T : 1) : bal_chunk(T, E, n_seq);
  const int chunks = bal_chunks(T, chunk);
  const int extra = (T > 0 ? chunks : 0) + 1;   // one workgroup counts the non-empty sequences
  bal_shape(E, [&](auto g, auto vec) {
    constexpr int G = decltype(g)::value;
    constexpr bool VEC = decltype(vec)::value;
    const auto kernel = one ? balance_chunk_kernel<G, VEC, true>
                            : balance_chunk_kernel<G, VEC, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(one ? 1 : extra)), dim3(kBalThreads), 0, s,
                       logits, topk_idx, alive, seq_offsets, T, E, k, n_seq, chunk, w, o);
  });
  if (one) return hipGetLastError();
  const bool few = n_seq * bal_blocks(E, kSumColsFew) <= kLastParts;
  const int blocks = bal_blocks(E, few ? kSumColsFew : kSumCols);
  hipLaunchKernelGGL(few ? balance_sum_kernel<kSumColsFew> : balance_sum_kernel<kSumCols>,
                     dim3((unsigned)n_seq, (unsigned)blocks), dim3(kSumThreads), 0, s, alive,
                     seq_offsets, T, E, k, n_seq, chunk, w, o);
  if (n_seq * blocks > kLastParts)
    hipLaunchKernelGGL(balance_loss_kernel, dim3(1), dim3(kWave), 0, s, w.part_loss,
                       n_seq * blocks, loss);
  return hipGetLastError();
}

hipError_t launch_balance_bwd(const float* logits, const float* grad_coef, const uint8_t* alive,
                              const int32_t* seq_offsets, const float* dloss, int T, int E,
                              int n_seq, float* dlogits, int accumulate, hipStream_t s) {
  if (T == 0) return hipSuccess;
  bal_shape(E, [&](auto g, auto vec) {
    constexpr int G = decltype(g)::value;
    constexpr int ROWS = kBalThreads / G;
    // one pass of the rows in flight, about two sequences at most; longer where the grid
    // would pass 2^14 workgroups
    const int least = bal_cut(ROWS * kBalAhead, T, n_seq), per = (T - 1) / (1 << 14) + 1;
    const int range = per > least ? per : least;
    hipLaunchKernelGGL((balance_bwd_kernel<G, decltype(vec)::value>),
                       dim3((unsigned)((T - 1) / range + 1)), dim3(kBalThreads), 0, s, logits,
                       grad_coef, alive, seq_offsets, dloss, T, E, n_seq, range, dlogits,
                       accumulate);
  });
  return hipGetLastError();
}

}  // namespace laep
