// Balance loss of the router (moe_balance_loss, moe_balance_loss_bwd).  With p the
// softmax of the alive experts' logits and the T tokens cut into sequences s of
// n_s tokens,
//   counts[s, e] = slots of s routed to e,  P[s, e] = mean over s of p[t, e],
//   f[s, e] = N_alive counts[s, e] / (k n_s),
//   loss = coef * mean over the non-empty s of sum_e f[s, e] P[s, e],
//   c[s, e] = coef f[s, e] / (n_s S_nonempty)     (= dloss / dp[t, e]),
//   dlogits[t, e] = dloss p_e (c_e - sum_i p_i c_i).
// The tokens are cut into equal chunks, one workgroup each, whatever the sequences:
// walking chunks and sequences in token order, each step goes to the next chunk or to
// the next sequence, so the pair (chunk c, sequence s) has the slot c + s to itself,
// and the partial sums need n_chunks + n_seq slots however the sequences fall.  A
// second pass sums each sequence's slots in order.  Counts are integers; every
// floating-point sum has a fixed order.
#include "common.hpp"
#include "internal.hpp"

namespace laep {
namespace {

constexpr int kBalThreads = 256;
constexpr int kBalWaves = kBalThreads / kWave;
constexpr int kBalMaxE = 256;
constexpr int kBalChunk = 64;      // tokens per workgroup, while that is
constexpr int kBalMaxChunks = 2048;  // at most so many workgroups
constexpr int kBalCols = 16;       // experts per workgroup of the second pass

struct BalWs {          // carved from the workspace
  int* live;            // non-empty sequences
  int* done;            // workgroups of the second pass that have finished
  float* part_p;        // [slots, E]
  int* part_n;          // [slots, E]
  float* part_loss;     // [n_seq, column blocks]
};

inline int bal_chunk(int T) {
  return T <= kBalChunk * kBalMaxChunks ? kBalChunk : (T - 1) / kBalMaxChunks + 1;
}
inline int bal_chunks(int T) { return T > 0 ? (T - 1) / bal_chunk(T) + 1 : 1; }
// chunks a workspace has to hold: grows with T, so that a workspace for the largest
// call serves the smaller ones (bal_chunks falls where a chunk gains a token)
inline int bal_chunks_bound(int T) {
  const int n = T > 0 ? (T - 1) / kBalChunk + 1 : 1;
  return n < kBalMaxChunks ? n : kBalMaxChunks;
}
inline int bal_blocks(int E) { return (E + kBalCols - 1) / kBalCols; }

inline size_t bal_carve(void* ws, int T, int E, int S, BalWs& w) {
  char* p = static_cast<char*>(ws);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* const r = p + at;
    at += align_up(bytes, 256);
    return r;
  };
  const size_t cells = ((size_t)bal_chunks_bound(T) + S) * E;
  w.live = reinterpret_cast<int*>(take(8));
  w.done = w.live + 1;
  w.part_p = reinterpret_cast<float*>(take(cells * 4));
  w.part_n = reinterpret_cast<int*>(take(cells * 4));
  w.part_loss = reinterpret_cast<float*>(take((size_t)S * bal_blocks(E) * 4));
  return at;
}

// Token range of sequence s (no offsets: one sequence of all tokens), inside [0, T].
__device__ __forceinline__ void seq_range(const int32_t* __restrict__ off, int s, int T, int& a,
                                          int& b) {
  a = off ? min(max(off[s], 0), T) : 0;
  b = off ? min(max(off[s + 1], a), T) : T;
}

// First sequence that ends after token t (n_seq if none does).
__device__ __forceinline__ int first_seq(const int32_t* __restrict__ off, int n_seq, int t) {
  if (!off) return 0;
  int lo = 0, hi = n_seq;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (off[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// One token's probabilities in a wave: lane l holds experts l, l + 64, ...  A token
// without an alive expert of finite or infinite logit gets zeros.
constexpr int kEpl = kBalMaxE / kWave;
__device__ __forceinline__ void token_probs(const float* __restrict__ row, int E, int lane,
                                            const bool alive[kEpl], float p[kEpl]) {
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < kEpl; ++u) {
    p[u] = alive[u] ? row[lane + kWave * u] : -INFINITY;
    m = fmaxf(m, p[u]);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
  const float base = m == -INFINITY ? 0.0f : m;
  float z = 0.0f;
#pragma unroll
  for (int u = 0; u < kEpl; ++u) {
    p[u] = expf(p[u] - base);
    z += p[u];
  }
  z = wave_sum(z);
  const float inv = z == 0.0f ? 0.0f : 1.0f / z;
#pragma unroll
  for (int u = 0; u < kEpl; ++u) p[u] *= inv;
}

__device__ __forceinline__ void load_alive(const uint8_t* __restrict__ alive, int E, int lane,
                                           bool a[kEpl]) {
#pragma unroll
  for (int u = 0; u < kEpl; ++u) {
    const int e = lane + kWave * u;
    a[u] = e < E && (alive == nullptr || alive[e] != 0);
  }
}

// First pass: chunk c's probability sums and counts of each sequence in it.
__global__ __launch_bounds__(kBalThreads) void balance_chunk_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ topk_idx,
    const uint8_t* __restrict__ alive, const int32_t* __restrict__ off, int T, int E, int k,
    int n_seq, int chunk, BalWs w) {
  __shared__ float s_p[kBalWaves][kBalMaxE];
  __shared__ int s_n[kBalMaxE];
  __shared__ int s_live;
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid & (kWave - 1);
  if (blockIdx.x == 0) {  // what the second pass needs once
    if (tid == 0) s_live = 0;
    __syncthreads();
    int n = 0;
    for (int s = tid; s < n_seq; s += kBalThreads) {
      int a, b;
      seq_range(off, s, T, a, b);
      n += b > a;
    }
    if (n) atomicAdd(&s_live, n);
    __syncthreads();
    if (tid == 0) {
      *w.live = s_live;
      *w.done = 0;
    }
  }
  bool ok[kEpl];
  load_alive(alive, E, lane, ok);
  const int t0 = blockIdx.x * chunk, t1 = T - t0 < chunk ? T : t0 + chunk;
  for (int s = first_seq(off, n_seq, t0); s < n_seq; ++s) {
    int a, b;
    seq_range(off, s, T, a, b);
    if (a >= t1) break;
    a = max(a, t0);
    b = min(b, t1);
    if (a >= b) continue;  // (uniform)
    for (int e = tid; e < E; e += kBalThreads) s_n[e] = 0;
    __syncthreads();
    float sum[kEpl] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int t = a + wave; t < b; t += kBalWaves) {
      float p[kEpl];
      token_probs(logits + (size_t)t * E, E, lane, ok, p);
#pragma unroll
      for (int u = 0; u < kEpl; ++u) sum[u] += p[u];
    }
    for (size_t i = (size_t)a * k + tid; i < (size_t)b * k; i += kBalThreads) {
      const int e = topk_idx[i];
      if (e >= 0 && e < E) atomicAdd(&s_n[e], 1);
    }
#pragma unroll
    for (int u = 0; u < kEpl; ++u) s_p[wave][lane + kWave * u] = sum[u];
    __syncthreads();
    const size_t slot = ((size_t)blockIdx.x + s) * E;
    for (int e = tid; e < E; e += kBalThreads) {
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < kBalWaves; ++i) v += s_p[i][e];
      w.part_p[slot + e] = v;
      w.part_n[slot + e] = s_n[e];
    }
    __syncthreads();
  }
}

// Second pass: 16 experts of one sequence per workgroup, its chunks' sums in order;
// the workgroup that finishes last adds the loss's parts, in order.
__global__ __launch_bounds__(kBalThreads) void balance_finish_kernel(
    const uint8_t* __restrict__ alive, const int32_t* __restrict__ off, int T, int E, int k,
    int n_seq, int chunk, float coef, BalWs w, float* __restrict__ loss, int32_t* __restrict__ counts,
    float* __restrict__ prob_mean, float* __restrict__ grad_coef) {
  constexpr int ROWS = kBalThreads / kBalCols;
  __shared__ float s_p[ROWS][kBalCols];
  __shared__ int s_n[ROWS][kBalCols];
  __shared__ float s_l[kBalThreads];
  __shared__ int s_last;
  const int tid = threadIdx.x, col = tid % kBalCols, row = tid / kBalCols;
  const int s = blockIdx.x, e = blockIdx.y * kBalCols + col;
  const int n_alive = alive == nullptr ? E : __syncthreads_count(tid < E && alive[tid] != 0);
  int a, b;
  seq_range(off, s, T, a, b);
  float p = 0.0f;
  int n = 0;
  if (b > a && e < E)
    for (int c = a / chunk + row; c <= (b - 1) / chunk; c += ROWS) {
      const size_t at = ((size_t)c + s) * E + e;
      p += w.part_p[at];
      n += w.part_n[at];
    }
  s_p[row][col] = p;
  s_n[row][col] = n;
  __syncthreads();
  float part = 0.0f;
  if (row == 0 && e < E) {
    p = 0.0f;
    n = 0;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      p += s_p[i][col];
      n += s_n[i][col];
    }
    const size_t at = (size_t)s * E + e;
    float mean = 0.0f, c = 0.0f;
    if (b > a) {
      const float len = (float)(b - a);
      mean = p / len;
      const float f = (float)n_alive * (float)n / ((float)k * len);
      part = coef * f * mean / (float)*w.live;
      c = coef * f / (len * (float)*w.live);
    }
    counts[at] = n;
    prob_mean[at] = mean;
    grad_coef[at] = c;
  }
  s_l[tid] = part;
  __syncthreads();
  const int n_parts = gridDim.x * gridDim.y;
  if (tid == 0) {
    float v = 0.0f;
    for (int i = 0; i < kBalCols; ++i) v += s_l[i];
    __hip_atomic_store(&w.part_loss[(size_t)s * gridDim.y + blockIdx.y], v, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
    s_last = __hip_atomic_fetch_add(w.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) ==
             n_parts - 1;
  }
  __syncthreads();
  if (!s_last) return;
  float v = 0.0f;
  for (int i = tid; i < n_parts; i += kBalThreads)
    v += __hip_atomic_load(&w.part_loss[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  s_l[tid] = v;
  __syncthreads();
  if (tid < kWave) {
    v = 0.0f;
    for (int i = tid; i < kBalThreads; i += kWave) v += s_l[i];
    v = wave_sum(v);
    if (tid == 0) *loss = v;
  }
}

// One wave per token; tokens of no sequence get a zero gradient.
__global__ __launch_bounds__(kBalThreads) void balance_bwd_kernel(
    const float* __restrict__ logits, const float* __restrict__ grad_coef,
    const uint8_t* __restrict__ alive, const int32_t* __restrict__ off,
    const float* __restrict__ dloss, int T, int E, int n_seq, float* dlogits, int accumulate) {
  const int lane = threadIdx.x & (kWave - 1);
  bool ok[kEpl];
  load_alive(alive, E, lane, ok);
  const float scale = dloss ? *dloss : 1.0f;
  const int step = gridDim.x * kBalWaves;
  for (int t = blockIdx.x * kBalWaves + threadIdx.x / kWave; t < T; t += step) {
    const int s = first_seq(off, n_seq, t);
    bool in = s < n_seq;
    if (in) {
      int a, b;
      seq_range(off, s, T, a, b);
      in = t >= a;
    }
    float p[kEpl], c[kEpl];
    token_probs(logits + (size_t)t * E, E, lane, ok, p);
    float dot = 0.0f;
#pragma unroll
    for (int u = 0; u < kEpl; ++u) {
      c[u] = in && ok[u] ? grad_coef[(size_t)s * E + lane + kWave * u] : 0.0f;
      dot += p[u] * c[u];
    }
    dot = wave_sum(dot);
#pragma unroll
    for (int u = 0; u < kEpl; ++u) {
      const int e = lane + kWave * u;
      if (e >= E) continue;
      float* const o = dlogits + (size_t)t * E + e;
      const float v = in && ok[u] ? scale * p[u] * (c[u] - dot) : 0.0f;
      *o = accumulate ? *o + v : v;
    }
    if (T - t <= step) break;  // (t + step past int32)
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
  hipLaunchKernelGGL(balance_chunk_kernel, dim3((unsigned)bal_chunks(T)), dim3(kBalThreads), 0, s,
                     logits, topk_idx, alive, seq_offsets, T, E, k, n_seq, bal_chunk(T), w);
  hipLaunchKernelGGL(balance_finish_kernel, dim3((unsigned)n_seq, (unsigned)bal_blocks(E)),
                     dim3(kBalThreads), 0, s, alive, seq_offsets, T, E, k, n_seq, bal_chunk(T), coef, w, loss,
                     counts, prob_mean, grad_coef);
  return hipGetLastError();
}

hipError_t launch_balance_bwd(const float* logits, const float* grad_coef, const uint8_t* alive,
                              const int32_t* seq_offsets, const float* dloss, int T, int E,
                              int n_seq, float* dlogits, int accumulate, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const int n = (T - 1) / kBalWaves + 1;
  hipLaunchKernelGGL(balance_bwd_kernel, dim3((unsigned)(n < 1 << 16 ? n : 1 << 16)),
                     dim3(kBalThreads), 0, s, logits, grad_coef, alive, seq_offsets, dloss, T, E,
                     n_seq, dlogits, accumulate);
  return hipGetLastError();
}

}  // namespace laep
