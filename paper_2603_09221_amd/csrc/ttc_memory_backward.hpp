// What the gradients of linear attention need beside memory_chunk_kernel's: those of the log decays, and sums over heads that share a query.
//
// With <R_t, S_t> the product of a state and of the loss's gradient with respect to it, dl/dg_t = exp(g_t) <R_t, S_{t-1}>: what tokens before t
// put in, as far as tokens from t on read it.  Pairs of one chunk are added up one by one (no difference of large sums):
//     dl/dg_t = sum_{j < t <= i} m_ij + I + sum_{s < t} (b_s - a_s),      m_ij = scale exp(G_i - G_j) (q_i . k_j) (dout_i . v_j),
// the last sum over the earlier tokens of the segment: a_s is q_s times what dq_s has from the state before its chunk, b_s is k_s times what dk_s
// has from the state's gradient behind its chunk, I = <R, S> where the segment begins.  Sums over tokens are float64; their terms' errors of
// 2^-24 add up from one such beginning to the next.
#pragma once
#include "ttc_memory.hpp"

namespace ttc {

struct MemDecayArgs {
  MemSequences m;
  MemRows q, k, v, gout;
  int32_t heads, dk, dv, slices;
  float scale;
  const float* log_decay;
  int64_t g_token, g_head;
  float* pairs;                 // (heads, tokens)
  const float *a, *b;           // (slices, heads, tokens)
  MemStates begin;              // of the forward call
  const float* gstate;          // (sequences, heads, dk, dv), where a sequence began with a state
  const float *found, *found_r; // (entries, heads, dk, dv): the segments' states from before, and their gradients from behind
  float* out;                   // (tokens, heads), or
  double* sums;                 // (entries, heads): sums over tokens instead
};

// eight numbers of a row in memory, or zeros in their place
__device__ __forceinline__ srv_bf16x8 mem_global(const unsigned short* p, bool wanted) {
  MemEight<unsigned short> x;
  mem_fetch(p, x);
  return wanted ? __builtin_bit_cast(srv_bf16x8, x.x) : srv_bf16x8{};
}
__device__ __forceinline__ mem_float8 mem_global(const float* p, bool wanted) {
  MemEight<float> x;
  mem_fetch(p, x);
  if (!wanted) x = {};
  return {{x.x[0][0], x.x[0][1], x.x[0][2], x.x[0][3], x.x[1][0], x.x[1][1], x.x[1][2], x.x[1][3]}};
}

// The sum over sixteen lanes side by side, in each of them
template <int CTRL>
__device__ __forceinline__ float mem_dpp_add(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float mem_sixteen(float x) {
  x = mem_dpp_add<0xb1>(x);     // the neighbour's
  x = mem_dpp_add<0x4e>(x);     // of two
  x = mem_dpp_add<0x141>(x);    // mirrored: of four
  return mem_dpp_add<0x140>(x); // of eight
}

// sum_{j < t <= i} m_ij for the tokens t of one chunk of one head: its steps are column sums below and row sums left of the diagonal.  A wavefront has sixteen
// rows and the tiles of sixteen columns up to the diagonal, its operands from memory as they are; a block of entries of all of them is under way at once.
template <typename T>
__global__ void __launch_bounds__(256, 4) memory_pairs_kernel(const MemDecayArgs a) {
  typedef typename MemOperand<T>::type op_t;
  constexpr int STEPS = sizeof(T) == 2 ? 4 : 1;  // operands of 32 entries in a block: what registers hold
  __shared__ alignas(16) MemDecays dl;
  __shared__ alignas(16) float left[MEM_CHUNK], below[4][MEM_CHUNK];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  int64_t entry, seq, first;
  int head, none, chunk, n;
  mem_deal(a.m, blockIdx.x, a.heads, 1, entry, head, none);
  if (entry >= a.m.entries || !mem_segment(a.m, entry, seq, chunk, first, n)) return;
  const int64_t t0 = first + (int64_t)chunk * MEM_CHUNK;
  const int rows = min(MEM_CHUNK, n - chunk * MEM_CHUNK);
  if (rows <= 0) return;
  if (wave == 0) {
    mem_decays(lane < rows ? a.log_decay[(t0 + lane) * a.g_token + head * a.g_head] : 0.f, lane, false, 1.f, 1.f, dl);
  }
  srv_floatx4 z[2][4] = {};
  const int i = 16 * wave + c;
  // rows behind the last are read from it (their products have no place in a sum)
  const auto products = [&](const MemRows& late, const MemRows& early, srv_floatx4 (&to)[4]) {
    const T* x = static_cast<const T*>(late.p) + head / late.group * late.head + t0 * late.token + min(i, rows - 1) * (uint32_t)late.token;
    const T* y = static_cast<const T*>(early.p) + head / early.group * early.head + t0 * early.token;
    uint32_t at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = min(16 * j + c, rows - 1) * (uint32_t)early.token;
    for (int e0 = 0; e0 < late.d; e0 += 32 * STEPS) {
      op_t own[STEPS], other[STEPS][4];
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        const int e = e0 + 32 * s + 8 * g;
        const bool there = e < late.d;
        own[s] = mem_global(x + (there ? e : 0), there);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j <= wave) other[s][j] = mem_global(y + (at[j] + (there ? e : 0)), there);
      }
#pragma unroll
      for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j <= wave) to[j] = mem_mma(other[s][j], own[s], to[j]);
    }
  };
  products(a.q, a.k, z[0]);
  products(a.gout, a.v, z[1]);
  __syncthreads();
  const float own_hi = dl.hi[i], own_lo = dl.lo[i];
  float row = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    srv_floatx4 sums = {};
    if (j <= wave) {
      const srv_floatx4 hi = *reinterpret_cast<const srv_floatx4*>(&dl.hi[16 * j + 4 * g]), lo = *reinterpret_cast<const srv_floatx4*>(&dl.lo[16 * j + 4 * g]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = a.scale * z[0][j][r] * z[1][j][r] * mem_between(own_hi, own_lo, hi[r], lo[r], 1.f);
        asm volatile("" : "+v"(x));  // (a select, not a branch for every number)
        x = i < rows && 16 * j + 4 * g + r < i ? x : 0.f;
        row += x;
        sums[r] = mem_sixteen(x);
      }
    }
    if (c == 0) *reinterpret_cast<srv_floatx4*>(&below[wave][16 * j + 4 * g]) = sums;
  }
  row += __shfl_xor(row, 16, 64);
  row += __shfl_xor(row, 32, 64);
  if (g == 0) left[i] = row;
  __syncthreads();
  if (wave == 0) {
    const double step = (double)((below[0][lane] + below[1][lane]) + (below[2][lane] + below[3][lane])) - left[lane];
    const double sum = mem_sums(step) - step;
    if (lane < rows) a.pairs[head * a.m.tokens + t0 + lane] = (float)sum;
  }
}

constexpr int MEM_SUM_THREADS = 1024;

// One head of one segment: 1024 tokens at a time
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
      const double grad = a.pairs[t] + now + (sum - step);
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

static __global__ void memory_decay_sum_kernel(const double* sums, int64_t entries, int heads, float* out) {
  const int h = blockIdx.x * 64 + threadIdx.x;
  if (h >= heads) return;
  double x = 0.0;
  for (int64_t s = 0; s < entries; ++s) x += sums[s * heads + h];
  out[h] = (float)x;
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
