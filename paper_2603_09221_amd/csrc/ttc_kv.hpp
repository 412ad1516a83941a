// The paged key-value cache in 4 bits: new tokens into it with their positions (ttc_kv_append), and tokens out of it as numbers
// (ttc_kv_read).  Both are bound by memory: 16384 tokens of 32 query and 8 cache heads of 128 in 66 us (370 MB, 5.6 TB/s; with the
// queries written through the caches 15 us more), read back in 16 us.  Eight entries of a head to a thread, so that a thread's codes are
// one word and a block of 32 entries is four neighbouring lanes.  A workgroup takes consecutive tokens of one head: the pieces of the
// cache's lines that consecutive tokens fill (four tokens' values lie side by side) meet in one XCD's cache before they go to memory.
#pragma once
#include "ttc_serve.hpp"

namespace ttc {

struct KvAppendArgs {
  ttc_kv_append_t a;
  uint32_t cache_workgroups;         // that write the cache, ahead of those of the queries
  int q_pieces;                      // workgroups along the query heads: number i takes heads i, i + q_pieces, ..
  bool k_vec, v_vec, q_vec, qo_vec;  // rows that allow 16-byte accesses
  bool t_vec;                        // and the table's
};

// Cosines and sines of the pairs that entries e .. e+7 of a head belong to (half layout: pair of each entry; interleaved: four pairs)
struct KvTurn {
  float c[8], s[8];
};

template <bool HALF>
__device__ __forceinline__ KvTurn kv_turn(const float* row, int rot, int e, bool vec) {
  KvTurn t;
  constexpr int N = HALF ? 8 : 4;
  const int half = rot / 2;
  if (HALF ? (vec && half % 8 == 0) : (vec && rot % 8 == 0)) {
    if (e >= rot) return t;
    const srv_floatx4* cs = reinterpret_cast<const srv_floatx4*>(row + 2 * (HALF ? (e < half ? e : e - half) : e / 2));
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const srv_floatx4 q = cs[i];
      t.c[2 * i] = q[0]; t.s[2 * i] = q[1]; t.c[2 * i + 1] = q[2]; t.s[2 * i + 1] = q[3];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = HALF ? e + i : e + 2 * i;
      if (at >= rot) continue;
      const int pair = HALF ? (at < half ? at : at - half) : at / 2;
      t.c[i] = row[2 * pair];
      t.s[i] = row[2 * pair + 1];
    }
  }
  return t;
}

// Entries e .. e+7 of a head, as they lie in memory; and, where the pairs are a multiple of eight entries apart, their partners, which
// another lane of the wavefront has read.  (Past the caches' replacement, as the rotation reads, 16384 tokens took 79 us instead of 66.)
template <typename T>
struct KvRaw {
  float own[8];
  __device__ __forceinline__ void load(const float* p, bool vec) { srv_ld8(p, vec, own); }
  __device__ __forceinline__ void of_lane(int lane, float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __shfl(own[i], lane, 64);
  }
};
template <>
struct KvRaw<unsigned short> {
  srv_u16x8 own;
  __device__ __forceinline__ void load(const unsigned short* p, bool vec) { own = __builtin_bit_cast(srv_u16x8, srv_ld8_bf16(p, vec)); }
  __device__ __forceinline__ void of_lane(int lane, float (&x)[8]) const {
    typedef int four_t __attribute__((ext_vector_type(4)));
    four_t v = __builtin_bit_cast(four_t, own);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __shfl(v[i], lane, 64);
    const srv_u16x8 w = __builtin_bit_cast(srv_u16x8, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = srv_widen(w[i]);
  }
};

// The entries turned; `rot` is the same for all lanes, `turns` is false for those whose position is not in the table
template <typename T, bool HALF>
__device__ __forceinline__ void kv_turned(const KvRaw<T>& raw, const T* x, int rot, bool turns, int e, const KvTurn& t, float (&y)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = srv_widen(raw.own[i]);
  const int half = rot / 2, lane = threadIdx.x & 63;
  float partner[8];
  if (HALF && rot && half % 8 == 0) raw.of_lane(e < half ? lane + half / 8 : e < rot ? lane - half / 8 : lane, partner);
  if (e >= rot || !turns) return;
  if constexpr (!HALF) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + 2 * i < rot) {
        float a, b;
        srv_turn(y[2 * i], y[2 * i + 1], t.c[i], t.s[i], a, b);
        y[2 * i] = a;
        y[2 * i + 1] = b;
      }
  } else if (half % 8 == 0) {
    float other;
    if (e < half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) srv_turn(y[i], partner[i], t.c[i], t.s[i], y[i], other);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) srv_turn(partner[i], y[i], t.c[i], t.s[i], other, y[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = e + i;
      float other;
      if (at < half) srv_turn(y[i], srv_widen(x[at + half]), t.c[i], t.s[i], y[i], other);
      else if (at < rot) srv_turn(srv_widen(x[at - half]), y[i], t.c[i], t.s[i], other, y[i]);
    }
  }
}

// Codes of eight entries and the exponent byte of the block that they share with the other three lanes of the four.  The largest
// magnitude is found among the bits, where a NaN is larger than every number.  The exponent stops at 252, from where on 6 is the largest
// finite number's own (the code for 8 would be infinite).  Scaling by a power of two is exact; the conversion then rounds to nearest even
// and stops at 6.
__device__ __forceinline__ uint32_t kv_quantise(const float (&x)[8], uint32_t& e) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    m = b > m ? b : m;
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    const uint32_t b = __shfl_xor(m, o, 64);
    m = b > m ? b : m;
  }
  const uint32_t k = (m + 0x200000u) >> 23;  // the exponent, one more from 1.75 on
  const uint32_t b = k < 2 ? 0u : k - 2 < KV_LARGEST ? k - 2 : KV_LARGEST;
  const float inverse = __uint_as_float((254u - b) << 23);
  e = m >= 0x7f800000u ? 255u : b;
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0] * inverse, x[1] * inverse, 1.f, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2] * inverse, x[3] * inverse, 1.f, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4] * inverse, x[5] * inverse, 1.f, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6] * inverse, x[7] * inverse, 1.f, 3);
  return code;
}

template <int D>
struct KvPlace {  // of entries 8u .. 8u+7 of one token in one head of one page
  uint32_t codes_k, codes_v, exp_k, exp_v;
  __device__ __forceinline__ KvPlace(int t, int u, int page) {
    typedef KvParts<D> P;
    codes_k = t * P::TOKEN + 4 * u;
    // lane l holds entries l*D/16 ..: a thread's eight entries are two lanes' (D = 64), one lane's, or half of one's (D = 256)
    constexpr int LANES = P::LANE < 4 ? 4 / P::LANE : 1, PARTS = P::LANE > 4 ? P::LANE / 4 : 1;
    codes_v = P::values(page) + (uint32_t)(t / 4) * (16 * 4 * P::LANE) + (u * LANES / PARTS) * (4 * P::LANE) + (t % 4) * P::LANE + (u % PARTS) * 4;
    exp_k = P::key_exps(page) + t * P::BLOCKS + u / 4;
    exp_v = P::value_exps(page) + (uint32_t)(t / 4) * (4 * P::BLOCKS) + (u / 4) * 4 + t % 4;
  }
};

constexpr int KV_MANY = 4;  // query heads, or tokens of a cache head, that a thread takes where there is enough work for it

// Workgroups first of the cache's heads, then of the queries'.  Of the cache a workgroup takes N * 256/U tokens of one head; neighbouring workgroups
// take other heads, so that (with a multiple of eight of them) a head's pages are all written through one XCD's cache, where the parts of a line
// that two workgroups write come together.
template <typename T, int D, bool HALF, int N>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvAppendArgs p) {
  constexpr int U = D / 8, TOKENS = 256 / U;
  const ttc_kv_append_t& a = p.a;
  const int u = threadIdx.x % U, e = 8 * u, heads = a.cache.heads;
  if (blockIdx.x >= p.cache_workgroups) {
    // Eight groups of tokens side by side, the pieces of a group one after the other: an XCD reads a token's cosines once (16384 tokens of 32
    // heads 73 -> 67 us).
    const uint32_t b = blockIdx.x - p.cache_workgroups, groups = (uint32_t)((a.tokens + TOKENS - 1) / TOKENS);
    const uint32_t eight = b / (8 * p.q_pieces) * 8, wide = min(8u, groups - eight), r = b - eight * p.q_pieces;
    const int piece = r / wide;
    const int64_t token = (int64_t)(eight + r % wide) * TOKENS + threadIdx.x / U;
    if (token >= a.tokens) return;
    const int64_t pos = a.rot ? a.positions[token] : 0;
    const bool lost = (pos < 0 || pos >= a.table_rows) && e < a.rot;
    // all heads' reads are done before the first is written: in place a pair's two threads, of one wavefront, may read each other's entries
    KvRaw<T> raw[N];
    const T* x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int h = min(piece + i * p.q_pieces, a.heads_q - 1);
      x[i] = static_cast<const T*>(a.q) + token * a.q_token + (int64_t)h * a.q_head;
      raw[i].load(x[i] + e, p.q_vec);
    }
    KvTurn t;
    if (a.rot && !lost) t = kv_turn<HALF>(a.table + pos * a.rot, a.rot, e, p.t_vec);
    float y[N][8];
#pragma unroll
    for (int i = 0; i < N; ++i) kv_turned<T, HALF>(raw[i], x[i], a.rot, !lost, e, t, y[i]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int h = piece + i * p.q_pieces;
      if (h >= a.heads_q) break;
      if (lost) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[i][k] = e + k < a.rot ? __builtin_nanf("") : y[i][k];
      }
      T* const to = static_cast<T*>(a.q_out) + token * a.q_out_token + (int64_t)h * a.q_out_head + e;
      if constexpr (N > 1) srv_stream8(to, p.qo_vec, y[i]);
      else srv_st8(to, p.qo_vec, y[i]);
    }
    return;
  }
  const int piece = blockIdx.x % (2 * heads), h = piece >> 1;
  const bool value = piece & 1;
  const int64_t first = (int64_t)(blockIdx.x / (2 * heads)) * (N * TOKENS) + threadIdx.x / U;
  const int page = a.cache.page, log_page = __builtin_ctz(page);
  KvRaw<T> raw[N];
  const T* x[N];
  int64_t slot[N], pos[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t token = min(first + i * TOKENS, a.tokens - 1);
    slot[i] = first + i * TOKENS < a.tokens ? a.slots[token] : -1;
    pos[i] = !value && a.rot ? a.positions[token] : 0;
    x[i] = value ? static_cast<const T*>(a.v) + token * a.v_token + (int64_t)h * a.v_head
                 : static_cast<const T*>(a.k) + token * a.k_token + (int64_t)h * a.k_head;
    raw[i].load(x[i] + e, value ? p.v_vec : p.k_vec);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool lost = !value && (pos[i] < 0 || pos[i] >= a.table_rows) && e < a.rot;
    const int rot = value ? 0 : a.rot;
    KvTurn t;
    if (rot && !lost) t = kv_turn<HALF>(a.table + pos[i] * rot, rot, e, p.t_vec);
    float y[8];
    kv_turned<T, HALF>(raw[i], x[i], rot, !lost, e, t, y);
    if (lost) y[0] = __builtin_nanf("");
    uint32_t exp;
    const uint32_t code = kv_quantise(y, exp);
    if (slot[i] < 0 || slot[i] >= a.cache.pages * page) continue;
    unsigned char* base = static_cast<unsigned char*>(a.cache.data) + ((slot[i] >> log_page) * heads + h) * (int64_t)KvParts<D>::bytes(page);
    const KvPlace<D> at((int)(slot[i] & (page - 1)), u, page);
    if (!value) {
      *reinterpret_cast<uint32_t*>(base + at.codes_k) = code;
    } else if constexpr (D == 64) {  // two lanes' shares of two bytes
      *reinterpret_cast<unsigned short*>(base + at.codes_v) = (unsigned short)code;
      *reinterpret_cast<unsigned short*>(base + at.codes_v + 4 * KvParts<D>::LANE) = (unsigned short)(code >> 16);
    } else {
      *reinterpret_cast<uint32_t*>(base + at.codes_v) = code;
    }
    if (u % 4 == 0) base[value ? at.exp_v : at.exp_k] = (unsigned char)exp;
  }
}

// eight entries from their codes
__device__ __forceinline__ void kv_numbers(uint32_t code, uint32_t e, float (&x)[8]) {
  const float scale = e > KV_LARGEST ? __builtin_nanf("") : e == 0 ? __uint_as_float(0x00400000u) : srv_scale(e);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = (code >> (4 * i)) & 15, m = c & 7;
    // magnitudes 0 .5 1 1.5 2 3 4 6: exponent and mantissa of a float32, apart from the first two
    const float v = m < 2 ? 0.5f * m : __uint_as_float(0x3f800000u + ((m - 2) << 22));
    x[i] = (c & 8 ? -v : v) * scale;
  }
}

// STREAM: results larger than what the caches would keep
template <typename T, int D, bool STREAM>
__global__ void __launch_bounds__(256) kv_read_kernel(const ttc_kv_cache_t c, const int64_t* slots, int64_t n, T* k, T* v) {
  constexpr int U = D / 8;
  const int u = threadIdx.x % U, h = blockIdx.y, page = c.page, log_page = __builtin_ctz(page);
  const int64_t token = (int64_t)blockIdx.x * (256 / U) + threadIdx.x / U;
  if (token >= n) return;
  const int64_t slot = slots[token], row = (token * c.heads + h) * D + 8 * u;
  float x[8] = {}, y[8] = {};
  if (slot >= 0 && slot < c.pages * page) {
    const unsigned char* base = static_cast<const unsigned char*>(c.data) + ((slot >> log_page) * c.heads + h) * (int64_t)KvParts<D>::bytes(page);
    const KvPlace<D> at((int)(slot & (page - 1)), u, page);
    if (k) kv_numbers(*reinterpret_cast<const uint32_t*>(base + at.codes_k), base[at.exp_k], x);
    if (v) {
      uint32_t code;
      if constexpr (D == 64)
        code = *reinterpret_cast<const unsigned short*>(base + at.codes_v) |
               (uint32_t)*reinterpret_cast<const unsigned short*>(base + at.codes_v + 4 * KvParts<D>::LANE) << 16;
      else
        code = *reinterpret_cast<const uint32_t*>(base + at.codes_v);
      kv_numbers(code, base[at.exp_v], y);
    }
  }
  if constexpr (STREAM) {
    if (k) srv_stream8(k + row, true, x);
    if (v) srv_stream8(v + row, true, y);
  } else {
    if (k) srv_st8(k + row, true, x);
    if (v) srv_st8(v + row, true, y);
  }
}

}  // namespace ttc
