// What the gradients of linear attention need beside memory_chunk_kernel's: those of the log decays, and sums over heads that share a query.
//
// With <R_t, S_t> the product of a state and of the loss's gradient with respect to it, dl/dg_t = exp(g_t) <R_t, S_{t-1}>: what tokens before t
// put in, as far as tokens from t on read it.  Pairs of one chunk are added up one by one (MEM_OUT_PAIRS; no difference of large sums):
//     dl/dg_t = sum_{j < t <= i} m_ij + I + sum_{s < t} (b_s - a_s),      m_ij = scale exp(G_i - G_j) (q_i . k_j) (dout_i . v_j),
// the last sum over the earlier tokens of the segment: a_s is q_s times what dq_s has from the state before its chunk, b_s is k_s times what dk_s
// has from the state's gradient behind its chunk, I = <R, S> where the segment begins.  Sums over tokens are float64; their terms' errors of
// 2^-24 add up from one such beginning to the next.  A token whose exp(g) is 0 in float32 has the gradient 0, which the sum's terms would only come near to.
#pragma once
#include "ttc_memory.hpp"

namespace ttc {

struct MemDecayArgs {
  MemSequences m;
  int32_t heads, dk, dv, slices, pair_slices;
  const float* pairs;           // (pair_slices, heads, tokens): sum_{j < t <= i} m_ij of a chunk's pairs
  const float *a, *b;           // (slices, heads, tokens)
  const float* log_decay;
  int64_t g_token, g_head;
  MemStates begin;              // of the forward call
  const float* gstate;          // (sequences, heads, dk, dv), where a sequence began with a state
  const float *found, *found_r; // (entries, heads, dk, dv): the segments' states from before, and their gradients from behind
  float* out;                   // (tokens, heads), or
  double* sums;                 // (entries, heads): sums over tokens instead
};

constexpr int MEM_SUM_THREADS = 1024;
constexpr float MEM_FORGETS = -104.f;  // its exponential is less than half of float32's smallest number

// One head of one segment: 1024 tokens at a time.  Two states a segment are what it reads: 31 MB in 10 us for four times 2048 tokens of 16 heads of 128.
static __global__ void __launch_bounds__(MEM_SUM_THREADS) memory_decay_kernel(const MemDecayArgs a) {
  __shared__ double meet[2][MEM_SUM_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, head = blockIdx.x % a.heads;
  const int64_t entry = blockIdx.x / a.heads, size = (int64_t)a.dk * a.dv;
  int64_t seq, first;
  int segment, n;
  if (!mem_segment(a.m, entry, seq, segment, first, n)) {
    if (a.sums && tid == 0) a.sums[entry * a.heads + head] = 0.0;
    return;
  }
  const int t0 = segment * a.m.segment * MEM_CHUNK, t1 = (int)min((int64_t)t0 + (int64_t)a.m.segment * MEM_CHUNK, (int64_t)n);
  const auto whole = [&](double x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) meet[0][wave] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < MEM_SUM_THREADS / 64; ++w) x += meet[0][w];
    return x;
  };
  const float *s = nullptr, *r = nullptr;
  if (segment) {
    s = a.found + (entry * a.heads + head) * size;
    r = a.found_r + ((entry - 1) * a.heads + head) * size;
  } else if (const int64_t row = mem_begin(a.begin, seq, n); row >= 0) {
    s = a.begin.in + (row * a.heads + head) * size;
    r = a.gstate + (seq * a.heads + head) * size;
  }
  double now = 0.0;
  if (s) {
    for (int64_t e = tid * 4; e < size; e += MEM_SUM_THREADS * 4) {
      const srv_floatx4 x = *reinterpret_cast<const srv_floatx4*>(s + e), y = *reinterpret_cast<const srv_floatx4*>(r + e);
#pragma unroll
      for (int k = 0; k < 4; ++k) now += (double)x[k] * y[k];
    }
    now = whole(now);
  }
  double total = 0.0;
  for (int at = t0; at < t1; at += MEM_SUM_THREADS) {
    const int64_t t = head * a.m.tokens + first + at + tid;
    const bool real = at + tid < t1;
    double step = 0.0;
    if (real)
      for (int s = 0; s < a.slices; ++s) step += (double)a.b[s * a.heads * a.m.tokens + t] - a.a[s * a.heads * a.m.tokens + t];
    double sum = mem_sums(step);
    __syncthreads();
    if (lane == 63) meet[1][wave] = sum;
    __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < MEM_SUM_THREADS / 64; ++w) {
      const double x = meet[1][w];
      sum += w < wave ? x : 0.0;
      all += x;
    }
    if (real) {
      double grad = now + (sum - step);
      for (int s = 0; s < a.pair_slices; ++s) grad += a.pairs[s * a.heads * a.m.tokens + t];
      if (a.log_decay[(first + at + tid) * a.g_token + head * a.g_head] < MEM_FORGETS) grad *= 0.0;  // (NaN stays)
      if (a.out) a.out[(first + at + tid) * a.heads + head] = (float)grad;
      total += grad;
    }
    now += all;
  }
  if (a.sums) {
    total = whole(total);
    if (tid == 0) a.sums[entry * a.heads + head] = total;
  }
}

// A head to a workgroup, a share of the segments to a thread, in an order that depends on their number alone.  One thread that adds them all took as long
// as the rest of the call where sequences are many: gradients of 8192 times 8 tokens of 4 heads of 64 1304 us, so 2217.
static __global__ void __launch_bounds__(256) memory_decay_sum_kernel(const double* sums, int64_t entries, int heads, float* out) {
  __shared__ double meet[256];
  double x = 0.0;
#pragma unroll 4
  for (int64_t s = threadIdx.x; s < entries; s += 256) x += sums[s * heads + blockIdx.x];
  meet[threadIdx.x] = x;
  for (int n = 128; n; n >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < n) meet[threadIdx.x] += meet[threadIdx.x + n];
  }
  if (threadIdx.x == 0) out[blockIdx.x] = (float)meet[0];
}

// The gradients of heads that share a row, in their order: a chunk's tokens of one shared head to a workgroup, four entries at a time to a thread
template <typename T>
__global__ void __launch_bounds__(256) memory_heads_kernel(const MemSequences m, const float* parts0, T* out0, const float* parts1, T* out1, uint32_t split, int heads, int group, int d) {
  const bool second = blockIdx.x >= split;  // (two in one launch, as MemTwo)
  const float* const parts = second ? parts1 : parts0;
  T* const out = second ? out1 : out0;
  int64_t entry, seq, first;
  int head, none, chunk, n;
  mem_deal(m, second ? blockIdx.x - split : blockIdx.x, heads, 1, entry, head, none);
  if (entry >= m.entries || !mem_segment(m, entry, seq, chunk, first, n)) return;
  const int64_t t0 = first + (int64_t)chunk * MEM_CHUNK;
  const int quads = min(MEM_CHUNK, n - chunk * MEM_CHUNK) * (d / 4);
  for (int i = threadIdx.x; i < quads; i += 256) {
    const int64_t row = (t0 + i / (d / 4)) * heads + head;
    const int e = i % (d / 4) * 4;
    srv_floatx4 x = {};
    for (int h = 0; h < group; ++h) x += *reinterpret_cast<const srv_floatx4*>(parts + (row * group + h) * d + e);
    mem_out4(out + row * d + e, x);
  }
}

}  // namespace ttc
