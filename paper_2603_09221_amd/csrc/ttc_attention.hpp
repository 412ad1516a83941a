// Attention over the cache in 4 bits (ttc_attention): out = softmax(scale q K^T) V, one pass over the context with the running maximum
// and sum of the softmax.
//
// A row is one new token of one query head; the rows of a tile read the same cache head.  Both products run on the matrix cores with the
// rows as columns: S^T = K Q^T (16 tokens x 16 rows) leaves in each lane four tokens' scores of one row, and these are what the
// lane has to hold for O^T = V^T P^T, whose sum runs over the tokens, if the tokens of two such tiles are taken in the order in which the
// lanes hold them.  So the weights never move between lanes, maxima and sums are the lane's own but for one exchange among four lanes,
// and rescaling is a product of the lane's own numbers.
#pragma once
#include "ttc_attention_plan.hpp"
#include "ttc_serve.hpp"

namespace ttc {

// The row tile of a workgroup: its sequence's numbers and this lane's row
struct AttTile {
  int len;          // tokens in the cache
  int rows;         // rows of the sequence
  int64_t first_q;  // row of q of its first new token
  int first, last;  // tokens that the lane's row sees: first .. last (none where last < first)
  int lo, hi;       // all that the tile's rows see lies in lo .. hi-1
};

__device__ __forceinline__ AttTile att_tile(const AttentionArgs& p, int64_t seq, int tile, int row) {
  const ttc_attention_t& a = p.a;
  AttTile t;
  int64_t q0 = seq, q1 = seq + 1;
  if (a.cu_q) { q0 = a.cu_q[seq]; q1 = a.cu_q[seq + 1]; }
  q0 = q0 < 0 ? 0 : q0;
  q1 = q1 > a.tokens ? a.tokens : q1;
  int64_t m = q1 - q0;
  const int64_t all = m;  // (positions count every new token, also those behind max_q)
  m = m < 0 ? 0 : m > a.max_q ? a.max_q : m;
  int len = a.kv_len[seq];
  t.len = len < 0 ? 0 : len > a.max_kv ? a.max_kv : len;
  t.rows = (int)m * p.group;
  t.first_q = q0;
  const int r = tile * ATT_ROWS + row;
  const int r1 = min(t.rows, (tile + 1) * ATT_ROWS) - 1;  // last row of the tile
  const int shift = t.len - (int)all;                     // token number of the first new one
  if (a.causal) {
    t.last = min(shift + r / p.group, t.len - 1);
    t.first = a.window ? max(t.last - a.window + 1, 0) : 0;
    t.hi = min(shift + r1 / p.group, t.len - 1) + 1;
    t.lo = a.window ? max(min(shift + tile * ATT_ROWS / p.group, t.len - 1) - a.window + 1, 0) : 0;
  } else {
    t.last = t.len - 1;
    t.first = 0;
    t.hi = t.len;
    t.lo = 0;
  }
  if (r >= t.rows) t.last = -1;
  if (r1 < tile * ATT_ROWS) t.hi = 0;
  t.lo = t.lo / ATT_STEP * ATT_STEP;
  return t;
}

// A float32 number as the sum of TERMS bfloat16 ones: one, rounded, or three that give every bit
template <int TERMS>
__device__ __forceinline__ void att_split(float x, __bf16 (&t)[TERMS]) {
#pragma unroll
  for (int i = 0; i < TERMS; ++i) {
    t[i] = static_cast<__bf16>(x);
    x -= static_cast<float>(t[i]);
  }
}

// Eight codes (a word) to eight bfloat16 numbers, exactly: a code has two significant bits, the scale is a power of two
__device__ __forceinline__ srv_bf16x8 att_widen(uint32_t code, float scale) {
  const srv_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1),
                   c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return srv_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 128 in every byte that is 255
__device__ __forceinline__ uint32_t att_full_bytes(uint32_t x) { return x & ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

template <typename T, int D>
__global__ void __launch_bounds__(64 * ATT_WAVES) attention_kernel(const AttentionArgs p) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int TERMS = BF16 ? 1 : 3;   // bfloat16 parts of a query and of a weight
  constexpr int KS = D / 32;            // products of 32 entries that a score takes
  constexpr int KW = D / 32;            // words of codes of a lane's share of a key: D/4 entries
  constexpr int E = D / 16;             // entries of a value that a lane holds
  constexpr int VW = D / 32;            // words of four tokens' values of one lane
  typedef KvParts<D> P;
  typedef uint32_t kw_t __attribute__((ext_vector_type(KW)));
  typedef uint32_t vw_t __attribute__((ext_vector_type(VW)));
  const ttc_attention_t& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  const int span = blockIdx.x % p.spans;
  const int64_t item = blockIdx.x / p.spans;
  const int tile = (int)(item % p.row_tiles), head = (int)(item / p.row_tiles % a.cache.heads);
  const int64_t seq = item / p.row_tiles / a.cache.heads;
  const AttTile t = att_tile(p, seq, tile, c);
  const int begin = t.lo + span * p.span, end = min(t.hi, begin + p.span);
  if (span > 0 && begin >= end) return;  // (the whole workgroup: nothing reads what this span would have written)

  // the lane's share of its row: entries g*D/4 .. of every part
  srv_bf16x8 q[TERMS][KS];
  {
    const int r = tile * ATT_ROWS + c;
    const bool real = r < t.rows;
    const T* x = static_cast<const T*>(a.q) + (real ? (t.first_q + r / p.group) * a.q_token + (int64_t)(head * p.group + r % p.group) * a.q_head : 0) + g * (D / 4);
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
  srv_floatx4 o[E] = {};
  float m = -INFINITY, l = 0.f;
  const float to_log2 = a.scale * 1.44269504088896340736f;
  const int log_page = __builtin_ctz(a.cache.page), page_bytes = P::bytes(a.cache.page);
  const int32_t* pages = a.block_table + seq * a.table_stride;
  const unsigned char* cache = static_cast<const unsigned char*>(a.cache.data);

  for (int n0 = begin + wave * ATT_STEP; n0 < end; n0 += ATT_STEP * ATT_WAVES) {
    const unsigned char* base[4];
    int in[4];      // token of the page that the sixteen begin with
    bool there[4];  // whether the sixteen are in the cache at all
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + 16 * i;
      const int page = n < end ? pages[n >> log_page] : -1;
      there[i] = page >= 0 && page < a.cache.pages;
      in[i] = n & (a.cache.page - 1);
      base[i] = cache + ((int64_t)(there[i] ? page : 0) * a.cache.heads + head) * page_bytes;
    }
    // scores: S^T = K Q^T, sixteen tokens at a time
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int token = in[i] + c;
      const kw_t code = *reinterpret_cast<const kw_t*>(base[i] + token * P::TOKEN + g * (D / 8));
      const unsigned char* ke = base[i] + P::key_exps(a.cache.page) + token * P::BLOCKS;
      srv_floatx4 z = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const float scale = srv_scale(ke[(g * (D / 4) + 8 * k) / 32]);
        const srv_bf16x8 key = att_widen(code[k], scale);
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[x][k], z, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = n0 + 16 * i + 4 * g + j;
        s[i][j] = there[i] && n >= t.first && n <= t.last ? z[j] * to_log2 : -INFINITY;
      }
    }
    // running maximum and sum of the row: the lane's sixteen tokens, then the four lanes that share the row
    float top = m;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, s[i][j]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float zero = top == -INFINITY ? 0.f : top;  // (a row that has seen nothing yet)
    const float shrink = __builtin_amdgcn_exp2f(m - zero);
    m = top;
    l *= shrink;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] *= shrink;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = __builtin_amdgcn_exp2f(s[i][j] - zero);
        l += s[i][j];
      }
    // O^T += V^T P^T, 32 tokens at a time: lane (c, g) has tokens 4g .. 4g+3 of two sixteens
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      srv_bf16x8 w[TERMS];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        __bf16 part[TERMS];
        att_split<TERMS>(s[2 * h + k / 4][k % 4], part);
#pragma unroll
        for (int x = 0; x < TERMS; ++x) w[x][k] = part[x];
      }
      vw_t code[2];
      uint32_t exps[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int four = in[2 * h + i] / 4 + g;
        code[i] = *reinterpret_cast<const vw_t*>(base[2 * h + i] + P::values(a.cache.page) + (four * 16 + c) * (4 * P::LANE));
        exps[i] = *reinterpret_cast<const uint32_t*>(base[2 * h + i] + P::value_exps(a.cache.page) + (four * P::BLOCKS + c * E / 32) * 4);
      }
      // A weight of 0 takes out any number, but not NaN.  Blocks of NaN are rare: they are read as numbers, and what the rows that
      // see them get is made NaN by a product of its own.
      const uint32_t nan0 = att_full_bytes(exps[0]), nan1 = att_full_bytes(exps[1]);
      if (__builtin_amdgcn_ballot_w64((nan0 | nan1) != 0)) {
        srv_bf16x8 bad, seen;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int i = 2 * h + k / 4, n = n0 + 16 * i + 4 * g + k % 4;
          bad[k] = static_cast<__bf16>((k < 4 ? nan0 : nan1) >> (8 * (k % 4)) & 128 ? 1.f : 0.f);
          seen[k] = static_cast<__bf16>(there[i] && n >= t.first && n <= t.last ? 1.f : 0.f);
        }
        const srv_floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen, srv_floatx4{}, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < E; ++e) o[e][j] = hit[j] > 0.f ? __builtin_nanf("") : o[e][j];
        exps[0] ^= nan0;
        exps[1] ^= nan1;
      }
      srv_bf16x8 v[E];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float scale = srv_scale((exps[k / 4] >> (8 * (k % 4))) & 255);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          // token k % 4 of the four: E/2 bytes of codes each
          const int byte = (k % 4) * (E / 2) + e / 2;
          const uint32_t word = code[k / 4][byte / 4];
          srv_bf16x2 two;
          switch (byte % 4) {
            case 0: two = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0); break;
            case 1: two = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1); break;
            case 2: two = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2); break;
            default: two = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3); break;
          }
          v[e][k] = two[0];
          v[e + 1][k] = two[1];
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x) o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[e], w[x], o[e], 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  // the wavefronts' results join: lane (c, g) holds entries (4g + j)*E + e of row c
  __shared__ float part_o[ATT_WAVES][ATT_ROWS][D + 4];
  __shared__ float part_m[ATT_WAVES][ATT_ROWS], part_l[ATT_WAVES][ATT_ROWS];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < E; ++e) part_o[wave][c][(4 * g + j) * E + e] = o[e][j];
  if (g == 0) {
    part_m[wave][c] = m;
    part_l[wave][c] = l;
  }
  __syncthreads();
  const int row = threadIdx.x / 16, e0 = (threadIdx.x % 16) * E;
  float mm = -INFINITY, ll = 0.f, sum[E] = {};
#pragma unroll
  for (int w = 0; w < ATT_WAVES; ++w) mm = fmaxf(mm, part_m[w][row]);
  const float zero = mm == -INFINITY ? 0.f : mm;
#pragma unroll
  for (int w = 0; w < ATT_WAVES; ++w) {
    const float f = __builtin_amdgcn_exp2f(part_m[w][row] - zero);
    ll += f * part_l[w][row];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += f * part_o[w][row][e0 + e];
  }
  if (p.spans > 1) {
    float* stat = p.part_stat + (item * p.spans + span) * (2 * ATT_ROWS);
    float* out = p.part_out + ((item * p.spans + span) * ATT_ROWS + row) * D + e0;
    if (threadIdx.x % 16 == 0) {
      stat[row] = mm;
      stat[ATT_ROWS + row] = ll;
    }
#pragma unroll
    for (int e = 0; e < E; e += 4) *reinterpret_cast<srv_floatx4*>(out + e) = srv_floatx4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
    return;
  }
  const int r = tile * ATT_ROWS + row;
  if (r >= t.rows) return;
  const int64_t token = t.first_q + r / p.group;
  const int h = head * p.group + r % p.group;
  const float f = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
  T* y = static_cast<T*>(a.out) + token * a.out_token + (int64_t)h * a.out_head + e0;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = srv_narrow<T>(f * sum[e]);
  if (a.lse && threadIdx.x % 16 == 0) a.lse[token * a.heads_q + h] = (mm + __builtin_log2f(ll)) * 0.69314718055994530942f;
}

// The spans' results of one row tile
template <typename T, int D>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttentionArgs p) {
  constexpr int E = D / 16;
  const ttc_attention_t& a = p.a;
  const int64_t item = blockIdx.x;
  const int tile = (int)(item % p.row_tiles), head = (int)(item / p.row_tiles % a.cache.heads);
  const int64_t seq = item / p.row_tiles / a.cache.heads;
  const AttTile t = att_tile(p, seq, tile, 0);
  const int row = threadIdx.x / 16, e0 = (threadIdx.x % 16) * E, r = tile * ATT_ROWS + row;
  if (r >= t.rows) return;
  const int used = t.hi > t.lo ? (t.hi - t.lo + p.span - 1) / p.span : 0;
  const float* stat = p.part_stat + item * p.spans * (2 * ATT_ROWS);
  const float* part = p.part_out + item * p.spans * ATT_ROWS * D;
  float mm = -INFINITY, ll = 0.f, sum[E] = {};
  for (int s = 0; s < used; ++s) mm = fmaxf(mm, stat[s * 2 * ATT_ROWS + row]);
  const float zero = mm == -INFINITY ? 0.f : mm;
  for (int s = 0; s < used; ++s) {
    const float f = __builtin_amdgcn_exp2f(stat[s * 2 * ATT_ROWS + row] - zero);
    ll += f * stat[s * 2 * ATT_ROWS + ATT_ROWS + row];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += f * part[(s * ATT_ROWS + row) * D + e0 + e];
  }
  const int64_t token = t.first_q + r / p.group;
  const int h = head * p.group + r % p.group;
  const float f = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
  T* y = static_cast<T*>(a.out) + token * a.out_token + (int64_t)h * a.out_head + e0;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = srv_narrow<T>(f * sum[e]);
  if (a.lse && threadIdx.x % 16 == 0) a.lse[token * a.heads_q + h] = (mm + __builtin_log2f(ll)) * 0.69314718055994530942f;
}

}  // namespace ttc
