// Attention over the cache for many rows (ttc_attention of prompts and chunks of them): the products bound it, not the cache's bytes.
//
// As in attention_kernel the rows are the columns of both products, here of 32 x 32 x 16 tiles: S^T = K Q^T leaves in a lane sixteen tokens'
// scores of one row, and taking the tokens of O^T = V^T P^T in the order that the lanes hold them the weights never move.  A wavefront has
// 32 rows, a workgroup 128 of one cache head.  Keys are widened by each wavefront for itself, from codes that the first of them has brought
// into the compute unit's cache (32 bytes of codes widen to 128 of operand, so reading them widened from LDS would take four times the
// bytes, and that would be all the LDS can give).  Values have to be turned, four tokens' entries side by side, which costs an exchange per two
// entries: the workgroup does that once, into LDS, in the order of the lanes that read it, without bank conflicts.
#pragma once
#include "ttc_attention.hpp"

namespace ttc {

typedef float srv_floatx16 __attribute__((ext_vector_type(16)));

constexpr int PROMPT_ROWS = 32 * PROMPT_WAVES;  // rows of a workgroup

template <typename T, int D>
__global__ void __launch_bounds__(64 * PROMPT_WAVES, prompt_waves_per_simd(sizeof(T) == 2, D)) attention_prompt_kernel(const AttentionArgs p) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int TERMS = BF16 ? 1 : 3;
  constexpr int KS = D / 16;     // products of 16 entries that a score takes
  constexpr int KW = D / 16;     // words of codes of a lane's share of a key: D/2 entries
  constexpr int E = D / 16;      // entries of a value in one of the cache's 16 lanes
  constexpr int DT = D / 32;     // tiles of 32 entries
  constexpr int EXPS = D / 64;   // exponents of a lane's share of a key
  typedef KvParts<D> P;
  typedef uint32_t key_t __attribute__((ext_vector_type(KW)));
  typedef uint32_t val_t __attribute__((ext_vector_type(D / 32)));
  static_assert(ATT_STEP == 64 && PROMPT_WAVES == 4, "a step is four sixteens, a wavefront turns one");

  const ttc_attention_t& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, g = lane >> 5;
  // heads fastest: with a multiple of eight of them an XCD's cache holds the keys and values of its own; the tiles that see most first
  const int64_t item = blockIdx.x;
  const int head = (int)(item % a.cache.heads);
  const int64_t seq = item / a.cache.heads % a.sequences;
  const int tile = p.row_tiles - 1 - (int)(item / a.cache.heads / a.sequences);
  const AttTile t = att_tile<PROMPT_ROWS>(p, seq, tile, 32 * wave + c);
  if (!t.real) return;

  // values of a step, widened: [four tokens' place][entry's place][8 tokens], and their exponents; two steps
  __shared__ srv_bf16x8 turned[2][8][D];
  __shared__ uint32_t exps[2][16][D / 32];
  __shared__ int bad_step[2][PROMPT_WAVES];

  const int r = tile * PROMPT_ROWS + 32 * wave + c;
  const int64_t token = t.first_q + r / p.group;
  const int h = head * p.group + r % p.group;
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
        att_split<TERMS>(v[i], part);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) q[k][s][i] = part[k];
      }
    }
  }
  srv_floatx16 o[DT] = {};
  float m = -INFINITY, l = 0.f;
  const float to_log2 = a.scale * 1.44269504088896340736f;
  const AttSource src(p, seq, head, t.hi);

  // keys: lane (c, g) has entries g*D/2 .. of token c of each 32; values: thread (f, l) has those of four tokens f that the cache's lane l holds
  key_t key[2];
  uint32_t key_exp[2];
  val_t value;
  uint32_t value_exp;
  int page[4];
  const auto load_keys = [&](int n0) {
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
  const auto load_values = [&](int n0) {
    const unsigned char* base = src.base(wave == 0 ? page[0] : wave == 1 ? page[1] : wave == 2 ? page[2] : page[3]);
    const uint32_t four = ((n0 + 16 * wave) & (src.page_tokens - 1)) / 4 + (f & 3);
    value = *reinterpret_cast<const val_t*>(base + (P::values(src.page_tokens) + (four * 16 + vl) * (4 * P::LANE)));
    value_exp = *reinterpret_cast<const uint32_t*>(base + (P::value_exps(src.page_tokens) + (four * P::BLOCKS + vl * E / 32) * 4));
  };
  // Row 32*dt + i of O^T is entry (i % 16) * E + 2*dt + i / 16, so that the threads of a cache's lane write side by side
  const auto turn_values = [&](int buffer) {
    const uint32_t nan = att_full_bytes(value_exp);
    if (vl * E % 32 == 0) exps[buffer][f][vl * E / 32] = value_exp;
    const bool any = __builtin_amdgcn_ballot_w64(nan != 0) != 0;
    if (lane == 0) bad_step[buffer][wave] = any;
    const uint32_t finite = value_exp ^ nan;
    __bf16* const to = reinterpret_cast<__bf16*>(&turned[buffer][(f / 4) * 2 + (f & 1)][vl]) + (f & 2) * 2;
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

  int there = 0, buffer = 0;
  if (t.lo < t.hi) {
    src.look_up(t.lo, page);
    there = src.there(t.lo, page);
    load_keys(t.lo);
    load_values(t.lo);
    src.look_up(t.lo + ATT_STEP, page);
    turn_values(0);
  }
  __syncthreads();
  for (int n0 = t.lo; n0 < t.hi; n0 += ATT_STEP, buffer ^= 1) {
    const bool more = n0 + ATT_STEP < t.hi;
    if (more) load_values(n0 + ATT_STEP);
    srv_floatx16 z[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      z[u] = srv_floatx16{};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const srv_bf16x8 k = att_widen(key[u][s], srv_scale((key_exp[u] >> (8 * (s / 4))) & 255));
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) z[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[x][s], z[u], 0, 0, 0);
      }
    }
    const int now = there;
    if (more) {
      there = src.there(n0 + ATT_STEP, page);
      load_keys(n0 + ATT_STEP);
      src.look_up(n0 + 2 * ATT_STEP, page);
    }
    if (n0 < t.all_lo || n0 + ATT_STEP > t.all_hi || now != 15) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int n = n0 + 32 * u + 8 * (j / 4) + 4 * g + j % 4;
          z[u][j] = (now >> (2 * u + j / 8) & 1) && n >= t.first && n <= t.last ? z[u][j] * to_log2 : -INFINITY;
        }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) z[u] *= to_log2;
    }
    float top = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) top = fmaxf(top, z[u][j]);
    if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {  // (see attention_kernel)
      top = fmaxf(m, top);
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
      m = top;
      l *= shrink;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= shrink;
    }
    const float zero = m == -INFINITY ? 0.f : m;
    srv_bf16x8 w[TERMS][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float x = __builtin_amdgcn_exp2f(z[u][j] - zero);
        l += x;
        __bf16 part[TERMS];
        att_split<TERMS>(x, part);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) w[k][2 * u + j / 8][j % 8] = part[k];
      }
    if (bad_step[buffer][0] | bad_step[buffer][1] | bad_step[buffer][2] | bad_step[buffer][3]) {
      // blocks of NaN: what the rows that see them get is made NaN (see attention_kernel)
#pragma unroll 1
      for (int s = 0; s < 4; ++s) {
        srv_bf16x8 bad, seen;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int four = 4 * s + 2 * (k / 4) + g, n = n0 + 4 * four + k % 4;
          bad[k] = static_cast<__bf16>((exps[buffer][four][(c & 15) * E / 32] >> (8 * (k % 4)) & 255) == 255 ? 1.f : 0.f);
          seen[k] = static_cast<__bf16>((now >> s & 1) && n >= t.first && n <= t.last ? 1.f : 0.f);
        }
        const srv_floatx16 hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad, seen, srv_floatx16{}, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
          for (int i = 0; i < DT; ++i) o[i][j] = hit[j] > 0.f ? __builtin_nanf("") : o[i][j];
      }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const srv_bf16x8 v = turned[buffer][2 * s + g][32 * i + c];
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[x][s], o[i], 0, 0, 0);
      }
    if (more) turn_values(buffer ^ 1);
    __syncthreads();
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
    if constexpr (E >= 8) {
#pragma unroll
      for (int i = 0; i < E; i += 8) srv_st8(to + i, vec, reinterpret_cast<const float(&)[8]>(x[i]));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) to[i] = srv_narrow<T>(x[i]);
    }
  }
  if (a.lse && g == 0) a.lse[token * a.heads_q + h] = (m + __builtin_log2f(l)) * 0.69314718055994530942f;
}

}  // namespace ttc
