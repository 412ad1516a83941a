// Places of new tokens in a paged cache (ttc_kv_place): sums over the sequences' lengths, pages from and to a list, a slot for every token.
// A few kilobytes in and out: launches, and the chain of waits inside, are what it takes.  One workgroup adds up the sequences, 1024 at a
// time, and hands out the pages; the same workgroup, or where there are many tokens a launch of its own, finds each token's sequence by bisection.
#pragma once
#include "ttc_serve.hpp"

namespace ttc {

constexpr int PLACE_THREADS = 1024;       // sequences that are added up at once
// Tokens that the one workgroup places itself: 64 sequences with 2048 in 5.9 us, 9.1 with a second launch; with 4096 in 8.2 and 8.8, with 8192 in 12.7 and 8.9
constexpr int64_t PLACE_ALONE = 4096;
constexpr int PLACE_TOKENS = 4;           // tokens of a thread of place_tokens_kernel

// Inclusive sums over the workgroup's threads; every thread also gets the whole.  `waves`: 16 numbers of LDS, free again on return.
__device__ __forceinline__ int64_t place_sum(int64_t x, int64_t* waves, int64_t& whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    x += lane >= o ? y : 0;
  }
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  int64_t before = 0;
  whole = 0;
#pragma unroll
  for (int w = 0; w < PLACE_THREADS / 64; ++w) {
    const int64_t y = waves[w];
    before += w < wave ? y : 0;
    whole += y;
  }
  __syncthreads();
  return x + before;
}

// The last of n ascending numbers that is at most x (the first is)
template <typename T>
__device__ __forceinline__ int place_find(const T* at, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int64_t place_past(const ttc_kv_place_t& p, int64_t s) { return min(max(p.past[s], 0), (1 << 30) - 1); }
__device__ __forceinline__ int64_t place_pages(const ttc_kv_place_t& p, int64_t tokens) {
  return min((int64_t)(((uint32_t)tokens + p.page - 1) / (uint32_t)p.page), (int64_t)p.width);  // (tokens are below 2^31)
}

// Row t of sequence s, token `position` of it; s < 0: nobody's
__device__ __forceinline__ void place_token(const ttc_kv_place_t& p, int64_t t, int s, int64_t position) {
  int64_t slot = -1;
  if (s >= 0 && position < (int64_t)p.width * p.page) {
    const int32_t at = p.block_table[s * p.table_stride + (uint32_t)position / (uint32_t)p.page];
    if (at >= 0 && at < p.pages) slot = (int64_t)at * p.page + (uint32_t)position % (uint32_t)p.page;
  }
  p.slots[t] = slot;
  p.positions[t] = s < 0 ? 0 : position;
  if (p.sequence) p.sequence[t] = s;
}

__global__ void __launch_bounds__(PLACE_THREADS) place_sequences_kernel(const ttc_kv_place_t p, const bool tokens_too) {
  __shared__ int64_t waves[PLACE_THREADS / 64];
  __shared__ int64_t first[PLACE_THREADS + 1];     // rows of this turn's sequences, then their pages among those handed out
  __shared__ int64_t before[PLACE_THREADS];        // tokens that were there
  const int tid = threadIdx.x, lane = tid & 63;
  int64_t there = 0;
  if (p.free_pages) {
    there = min(max((int64_t)*p.free_count, (int64_t)0), p.free_capacity);
    // Ended sequences' pages: a wavefront goes through one table row after the other, 64 entries at a time.  Twice: how many there are has
    // to be known before the first is written.
    for (int64_t s0 = 0; s0 < p.sequences; s0 += PLACE_THREADS) {
      const int64_t s = s0 + tid;
      const bool ended = s < p.sequences && p.new_tokens[s] < 0;
      if (!__syncthreads_or(ended)) continue;
      const int held = ended ? (int)place_pages(p, place_past(p, s)) : 0;
      int64_t at = 0;
      const auto walk = [&](bool write) {
        int64_t valid = 0;
        for (uint64_t todo = __builtin_amdgcn_ballot_w64(ended); todo; todo &= todo - 1) {
          const int who = __builtin_ctzll(todo), n = __shfl(held, who, 64);
          const int32_t* row = p.block_table + (s0 + (tid & ~63) + who) * p.table_stride;
          const int64_t to = __shfl(at, who, 64);
          int64_t seen = 0;
          for (int c = 0; c < n; c += 64) {
            const int32_t page = c + lane < n ? row[c + lane] : -1;
            const bool good = page >= 0 && page < p.pages;
            const uint64_t all = __builtin_amdgcn_ballot_w64(good);
            const int64_t place = to + seen + __builtin_popcountll(all & ((1ull << lane) - 1));
            if (write && good && place < p.free_capacity) p.free_pages[place] = page;
            seen += __builtin_popcountll(all);
          }
          if (lane == who) valid = seen;
        }
        return valid;
      };
      const int64_t valid = walk(false);
      int64_t whole;
      at = there + place_sum(valid, waves, whole) - valid;
      walk(true);
      there = min(there + whole, p.free_capacity);
    }
    __syncthreads();  // the list is whole
  }
  int64_t rows = 0, given = 0;  // of the sequences of earlier turns
  for (int64_t s0 = 0; s0 < p.sequences; s0 += PLACE_THREADS) {
    const int64_t s = s0 + tid;
    const bool real = s < p.sequences;
    const int64_t asked = real ? p.new_tokens[s] : 0, past = real ? place_past(p, s) : 0;
    int64_t whole;
    const int64_t upto = min(rows + place_sum(max(asked, (int64_t)0), waves, whole), p.tokens);
    first[tid + 1] = upto;
    if (tid == 0) first[0] = rows;
    __syncthreads();
    const int64_t n = upto - first[tid];
    rows = min(rows + whole, p.tokens);
    if (real) {
      p.cu_q[s + 1] = (int32_t)upto;
      p.kv_len[s] = asked < 0 ? 0 : (int32_t)(past + n);
    }
    before[tid] = past;
    if (p.free_pages) {
      __syncthreads();
      const int64_t held = place_pages(p, past), lacks = real && asked >= 0 ? place_pages(p, past + n) - held : 0;
      const int64_t end = place_sum(lacks, waves, whole), mine = first[tid];
      first[tid] = end - lacks;
      if (tid == PLACE_THREADS - 1) first[PLACE_THREADS] = end;
      __syncthreads();
      for (int64_t i = tid; i < whole; i += PLACE_THREADS) {
        const int who = place_find(first, PLACE_THREADS, i);
        const int64_t k = given + i, column = place_pages(p, before[who]) + i - first[who];
        p.block_table[(s0 + who) * p.table_stride + column] = k < there ? p.free_pages[there - 1 - k] : -1;
      }
      given += whole;
      __syncthreads();
      first[tid] = mine;  // the rows again
      if (tid == 0) first[PLACE_THREADS] = rows;
    }
    if (tokens_too) {
      __syncthreads();
      for (int64_t t = first[0] + tid; t < rows; t += PLACE_THREADS) {
        const int who = place_find(first, PLACE_THREADS, t);
        place_token(p, t, (int)(s0 + who), before[who] + t - first[who]);
      }
    }
    __syncthreads();
  }
  if (tokens_too)
    for (int64_t t = rows + tid; t < p.tokens; t += PLACE_THREADS) place_token(p, t, -1, 0);
  if (tid == 0) {
    p.cu_q[0] = 0;
    if (p.free_pages) *p.free_count_out = (int32_t)max(there - given, (int64_t)0);
    if (p.missing) *p.missing = p.free_pages ? (int32_t)max(given - there, (int64_t)0) : 0;
  }
}

// Tokens after place_sequences_kernel.  Up to 1024 sequences' first rows are held in LDS.
__global__ void __launch_bounds__(256) place_tokens_kernel(const ttc_kv_place_t p) {
  __shared__ int32_t first[PLACE_THREADS + 1];
  const bool few = p.sequences <= PLACE_THREADS;
  if (few)
    for (int i = threadIdx.x; i <= (int)p.sequences; i += 256) first[i] = p.cu_q[i];
  __syncthreads();
  const int32_t* at = few ? first : p.cu_q;
  const int64_t rows = at[p.sequences];
#pragma unroll
  for (int i = 0; i < PLACE_TOKENS; ++i) {
    const int64_t t = ((int64_t)blockIdx.x * PLACE_TOKENS + i) * 256 + threadIdx.x;
    if (t >= p.tokens) return;
    if (t >= rows) {
      place_token(p, t, -1, 0);
    } else {
      const int s = place_find(at, (int)p.sequences, (int32_t)t);
      place_token(p, t, s, p.kv_len[s] - (at[s + 1] - t));
    }
  }
}

}  // namespace ttc
