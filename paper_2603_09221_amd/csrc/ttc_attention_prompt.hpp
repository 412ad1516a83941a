// Attention over the cache for many rows (ttc_attention of prompts and chunks of them): the products bound it, not the cache's bytes.
//
// As in attention_kernel the rows are the columns of both products, here of 32 x 32 x 16 tiles: S^T = K Q^T leaves in a lane sixteen tokens'
// scores of one row, and taking the tokens of O^T = V^T P^T in the order that the lanes hold them the weights never move.  A wavefront has
// 32 rows, a workgroup 128 of one cache head.  Keys are widened by each wavefront for itself (widened once for the workgroup, through LDS, every
// product waits for its operand: 838 us where this takes 700).  Values have to be turned, four tokens' entries side by side, which costs an
// exchange per two entries: the workgroup does that once, into LDS, in the order of the lanes that read it (a quarter of LDS's busy cycles are conflicts, of the writes; LDS is busy a quarter of the time).
//
// 4096 queries of 32 heads over 12288 tokens (d = 128, 8 cache heads): 718 us, 0.96 PFLOP/s, where a large matrix product of the library
// runs at 1.25.  Matrix and vector instructions of the two wavefronts of a SIMD share its time, about 42 % and 62 % of the cycles: a step of 64
// tokens is 32 products (1024 cycles), 32 exponentials and about 270 other vector instructions.  With d = 64 half the products stand beside
// the same softmax.  Weights of bfloat16 rows are rounded for their product, as in attention_kernel.
#pragma once
#include <type_traits>

#include "ttc_attention.hpp"

namespace ttc {

typedef float srv_floatx16 __attribute__((ext_vector_type(16)));

constexpr int PROMPT_ROWS = 32 * PROMPT_WAVES;  // rows of a workgroup

// The place of item `at` (of one head): false if there are fewer.  Every wavefront adds up the sequences' tiles for itself, a run of sequences to
// a lane.  Where all have the same number, the tiles that see most come first, and each round of them begins with another sequence, for the
// contexts' lengths may differ and eight sequences of one head would each stay on one XCD.  Otherwise one sequence after the other: workgroups
// without a tile, left between the others, would leave compute units idle: 8 prompts of 17 to 1500 tokens, 16 query heads of one cache head,
// d = 64, a window of 512, took 58 us where this takes 35.
__device__ __forceinline__ bool prompt_tile(const AttentionArgs& p, int64_t at, int lane, int64_t& seq, int& tile) {
  const int64_t n = p.a.sequences, run = (n + 63) / 64, first = min(lane * run, n), last = min(first + run, n);
  const auto tiles = [&](int64_t s) {
    if (!p.a.cu_q) return (uint32_t)p.row_tiles;
    const int64_t q0 = max(p.a.cu_q[s], 0), q1 = min((int64_t)p.a.cu_q[s + 1], p.a.tokens), m = min(q1 - q0, (int64_t)p.a.max_q);
    return m > 0 ? (uint32_t)((m * p.group + PROMPT_ROWS - 1) / PROMPT_ROWS) : 0u;
  };
  uint32_t own = 0;
  for (int64_t s = first; s < last; ++s) own += tiles(s);
  uint32_t sum = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(sum, o, 64);
    sum += lane >= o ? x : 0;
  }
  const uint32_t total = __builtin_amdgcn_readlane(sum, 63);
  if (at >= total) return false;
  if (total == (uint32_t)p.entries) {
    const int64_t turn = at / n;
    tile = p.row_tiles - 1 - (int)turn;
    seq = n % 2 ? at % n : (at + turn) % n;
    return true;
  }
  uint32_t before = sum - own;
  const int there = __builtin_ctzll(__builtin_amdgcn_ballot_w64(at >= before && at < before + own));
  before = __builtin_amdgcn_readlane(before, there);
  for (int s = there * (int)run;; ++s) {
    const uint32_t m = __builtin_amdgcn_readfirstlane(tiles(s));
    if (at < before + m || s + 1 >= n) {
      seq = __builtin_amdgcn_readfirstlane(s);
      tile = __builtin_amdgcn_readfirstlane((int)(before + m - 1 - at));  // what sees most first
      return true;
    }
    before += m;
  }
}

// Workgroups of a compute unit at once: as many as the registers of a wavefront allow without spilling
template <typename T, int D>
__global__ void __launch_bounds__(64 * PROMPT_WAVES, sizeof(T) == 2 && D == 64 ? 3 : 2) attention_prompt_kernel(const AttentionArgs p) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int TERMS = BF16 ? 1 : 3;
  constexpr int KS = D / 16;     // products of 16 entries that a score takes
  constexpr int KW = D / 16;     // words of codes of a lane's share of a key: D/2 entries
  constexpr int EXPS = D / 64;   // exponents of a lane's share of a key
  constexpr int E = D / 16;      // entries of a value in one of the cache's 16 lanes
  constexpr int DT = D / 32;     // tiles of 32 entries
  typedef KvParts<D> P;
  typedef uint32_t key_t __attribute__((ext_vector_type(KW)));
  typedef uint32_t val_t __attribute__((ext_vector_type(D / 32)));
  static_assert(ATT_STEP == 64 && PROMPT_WAVES == 4, "a step is four sixteens, a wavefront turns one");

  const ttc_attention_t& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, g = lane >> 5;
  // heads fastest: with a multiple of eight of them an XCD's cache holds the keys and values of its own
  const int head = (int)(blockIdx.x % a.cache.heads);
  int64_t seq;
  int tile;
  if (!prompt_tile(p, blockIdx.x / a.cache.heads, lane, seq, tile)) return;
  const AttTile t = att_tile<PROMPT_ROWS>(p, seq, tile, 32 * wave + c);
  if (!t.real) return;

  // two steps' values, widened, [16 tokens][8 of them][entry's place]: eight numbers that a lane takes at once; and their exponents
  __shared__ srv_bf16x8 turned[2][4][2][D];
  __shared__ uint32_t exps[2][16][D / 32];
  __shared__ int bad_step[2][PROMPT_WAVES];

  const int r = tile * PROMPT_ROWS + 32 * wave + c;
  const int64_t token = t.first_q + r / p.group;
  const int h = head * p.group + r % p.group;
  // Queries take the scale's sign, so that the largest scores are the largest products, and a scale of 0 altogether: masked products are -inf
  // before they meet to_log2, which therefore must not be 0.
  const float size = fabsf(a.scale) * 1.44269504088896340736f, to_log2 = size == 0.f ? 1.f : size;
  const float sign = size == 0.f ? 0.f : a.scale < 0.f ? -1.f : 1.f;
  srv_bf16x8 q[TERMS][KS];
  {
    const bool real = r < t.rows;
    const T* x = static_cast<const T*>(a.q) + (real ? token * a.q_token + (int64_t)h * a.q_head : 0) + g * (D / 2);
    const bool vec = (uint64_t)a.q % 16 == 0 && (a.q_token | a.q_head) % (16 / (int)sizeof(T)) == 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      float v[8] = {};
      if (real) srv_ld8(x + 8 * s, vec, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __bf16 part[TERMS];
        att_split<TERMS>(sign * v[i], part);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) q[k][s][i] = part[k];
      }
    }
  }
  srv_floatx16 o[DT] = {};
  float m = -INFINITY, l = 0.f;
  const AttSource src(p, seq, head, t.hi);

  // keys: lane (c, g) has entries g*D/2 .. of token c of each 32; values: thread (f, vl) has those of four tokens f that the cache's lane vl holds
  key_t key[2];
  uint32_t key_exp[2];
  val_t value;
  uint32_t value_exp;
  const auto load_keys = [&](int n0, const int (&page)[4]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const unsigned char* base = src.base(c < 16 ? page[2 * u] : page[2 * u + 1]);
      const uint32_t at = ((n0 + 32 * u + (c & 16)) & (src.page_tokens - 1)) + (c & 15);
      key[u] = *reinterpret_cast<const key_t*>(base + (at * P::TOKEN + g * (D / 4)));
      const unsigned char* e = base + (P::key_exps(src.page_tokens) + at * P::BLOCKS + g * EXPS);
      key_exp[u] = EXPS == 1 ? *e : EXPS == 2 ? *reinterpret_cast<const unsigned short*>(e) : *reinterpret_cast<const uint32_t*>(e);
    }
  };
  const int f = threadIdx.x >> 4, vl = threadIdx.x & 15;  // f / 4 is the wavefront's number
  const auto load_values = [&](int n0, const int (&page)[4]) {
    const unsigned char* base = src.base(wave == 0 ? page[0] : wave == 1 ? page[1] : wave == 2 ? page[2] : page[3]);
    const uint32_t four = ((n0 + 16 * wave) & (src.page_tokens - 1)) / 4 + (f & 3);
    value = *reinterpret_cast<const val_t*>(base + (P::values(src.page_tokens) + (four * 16 + vl) * (4 * P::LANE)));
    value_exp = *reinterpret_cast<const uint32_t*>(base + (P::value_exps(src.page_tokens) + (four * P::BLOCKS + vl * E / 32) * 4));
  };
  // Row 32*dt + i of O^T is entry (i % 16) * E + 2*dt + i / 16, so that the threads of the cache's lanes write side by side
  const auto turn_values = [&](int buffer) {
    const uint32_t nan = att_nan_bytes(value_exp);
    exps[buffer][f][vl * E / 32] = value_exp;  // (the same from all lanes of a block)
    bad_step[buffer][wave] = __builtin_amdgcn_ballot_w64(nan != 0) != 0;
    const uint32_t finite = value_exp ^ nan;
    __bf16* const to = reinterpret_cast<__bf16*>(&turned[buffer][wave][f & 1][vl]) + (f & 2) * 2;
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      typedef __bf16 four_t __attribute__((ext_vector_type(4)));
      four_t x, y;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const srv_bf16x2 two = att_value_pair<E>(value, k, e, srv_scale((finite >> (8 * k)) & 255));
        x[k] = two[0];
        y[k] = two[1];
      }
      *reinterpret_cast<four_t*>(to + e * 16 * 8) = x;
      *reinterpret_cast<four_t*>(to + (e + 1) * 16 * 8) = y;
    }
  };

  // Step n: beside the scores of its tokens, whose codes are widened on the way, values n are turned; beside the sum over the values of
  // step n-1 the weights of step n are formed.  The codes of step n+1 are on their way from memory meanwhile.
  srv_floatx16 z[2];        // products q . k, 32 tokens each
  srv_bf16x8 w[TERMS][4];   // weights, 16 tokens each
  int page[4], there = 0, there_before = 0;  // of step n+1; of steps n and n-1
  bool moved = false;
  float shrink = 1.f;
  const auto add_values = [&](int buffer) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const srv_bf16x8 v = turned[buffer][s][g][32 * i + c];
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[x][s], o[i], 0, 0, 0);
      }
  };
  // blocks of NaN among the values of the step from token n0 on: what the rows that see them get is made NaN (see attention_kernel)
  const auto spread_nan = [&](int n0, int buffer, int there) {
    if (!(bad_step[buffer][0] | bad_step[buffer][1] | bad_step[buffer][2] | bad_step[buffer][3])) return;
#pragma unroll 1
    for (int s = 0; s < 4; ++s) {
      srv_bf16x8 bad, seen;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int four = 4 * s + 2 * (k / 4) + g, n = n0 + 4 * four + k % 4;
        bad[k] = static_cast<__bf16>((exps[buffer][four][(c & 15) * E / 32] >> (8 * (k % 4)) & 255) > KV_LARGEST ? 1.f : 0.f);
        seen[k] = static_cast<__bf16>((there >> s & 1) && n >= t.first && n <= t.last ? 1.f : 0.f);
      }
      const srv_floatx16 hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad, seen, srv_floatx16{}, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i][j] = hit[j] > 0.f ? __builtin_nanf("") : o[i][j];
    }
  };
  const auto step = [&](int n0, int buffer, auto first_) {
    constexpr bool first = decltype(first_)::value;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      z[u] = srv_floatx16{};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const srv_bf16x8 k = att_widen(key[u][s], srv_scale_or_nan((key_exp[u] >> (8 * (s / 4))) & 255));
#pragma unroll
        for (int i = TERMS - 1; i >= 0; --i) z[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[i][s], z[u], 0, 0, 0);
      }
    }
    turn_values(buffer);
    // a product, then what else there is to do while it runs: about six vector instructions
    if constexpr (BF16) {
      __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
        __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
      }
    }
    load_keys(n0 + ATT_STEP, page);
    load_values(n0 + ATT_STEP, page);
    const int next = src.there(n0 + ATT_STEP, page);
    src.look_up(n0 + 2 * ATT_STEP, page);
    if (n0 < t.all_lo || n0 + ATT_STEP > t.all_hi || there != 15) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int n = n0 + 32 * u + 8 * (j / 4) + 4 * g + j % 4;
          z[u][j] = (there >> (2 * u + j / 8) & 1) && n >= t.first && n <= t.last ? z[u][j] : -INFINITY;
        }
    }
    // The weights of step n-1 are relative to that step's maximum
    if (moved) {
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= shrink;
    }
    // The maximum that weights are relative to (in units of log2) moves as attention_kernel's does
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, z[u][j]);
    top *= to_log2;
    moved = __builtin_amdgcn_ballot_w64(top > m + 8.f) != 0;
    if (moved) {
      top = fmaxf(m, top);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
      m = top;
      l *= shrink;
    }
    if constexpr (!first) spread_nan(n0 - ATT_STEP, buffer ^ 1, there_before);
    if constexpr (!first) add_values(buffer ^ 1);
    const float zero = m == -INFINITY ? 0.f : m;
    srv_bf16x8 w1[TERMS][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u][j], to_log2, -zero));
        l += x;
        __bf16 part[TERMS];
        att_split<TERMS>(x, part);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) w1[k][2 * u + j / 8][j % 8] = part[k];
      }
    if constexpr (BF16) {
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < TERMS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[k][i] = w1[k][i];
    there_before = there;
    there = next;
    __syncthreads();
  };

  if (t.lo < t.hi) {
    int n0 = t.lo, buffer = 0;
    src.look_up(n0, page);
    there = src.there(n0, page);
    load_keys(n0, page);
    load_values(n0, page);
    src.look_up(n0 + ATT_STEP, page);
    step(n0, 0, std::true_type{});
    for (n0 += ATT_STEP, buffer = 1; n0 < t.hi; n0 += ATT_STEP, buffer ^= 1) step(n0, buffer, std::false_type{});
    if (moved) {
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= shrink;
    }
    spread_nan(n0 - ATT_STEP, buffer ^ 1, there_before);
    add_values(buffer ^ 1);
  }
  l += __shfl_xor(l, 32, 64);
  if (r >= t.rows) return;
  // O^T's row 32*i + (j%4) + 8*(j/4) + 4*g: of the cache's lane vl all E entries are the lane's own, side by side
  const float inverse = l > 0.f || l != l ? 1.f / l : 0.f;
  T* y = static_cast<T*>(a.out) + token * a.out_token + (int64_t)h * a.out_head;
  const bool vec = (uint64_t)a.out % 16 == 0 && (a.out_token | a.out_head) % (16 / (int)sizeof(T)) == 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float x[E];
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      x[2 * i] = inverse * o[i][j];
      x[2 * i + 1] = inverse * o[i][j + 8];
    }
    T* const to = y + ((j % 4) + 8 * (j / 4) + 4 * g) * E;
    srv_st(to, vec, x);
  }
  if (a.lse && g == 0) a.lse[token * a.heads_q + h] = (m + __builtin_log2f(l)) * 0.69314718055994530942f;
}

}  // namespace ttc
