// The paged key-value cache in 4 bits: new tokens into it with their positions (ttc_kv_append), and tokens out of it as numbers
// (ttc_kv_read).  Both are bound by memory; eight entries of a head to a thread, so that a thread's codes are one word and a block of 32
// entries is four neighbouring lanes.  A workgroup takes consecutive tokens of one head: the pieces of the cache's lines that
// consecutive tokens fill (four tokens' values lie side by side) meet in one XCD's cache before they go to memory.
#pragma once
#include "ttc_serve.hpp"

namespace ttc {

struct KvAppendArgs {
  ttc_kv_append_t a;
  int q_pieces;                      // workgroups along the query heads, each of q_heads of them
  int q_heads;
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

// entries e .. e+7 of the head at x, turned
template <typename T, bool HALF>
__device__ __forceinline__ void kv_load_turned(const T* x, int rot, int e, bool vec, const KvTurn& t, float (&y)[8]) {
  srv_ld8(x + e, vec, y);
  if (e >= rot) return;
  const int half = rot / 2;
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
    float w[8], other;
    srv_ld8(x + (e < half ? e + half : e - half), vec, w);
    if (e < half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) srv_turn(y[i], w[i], t.c[i], t.s[i], y[i], other);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) srv_turn(w[i], y[i], t.c[i], t.s[i], other, y[i]);
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
  const uint32_t b = k < 2 ? 0u : k - 2 < 252u ? k - 2 : 252u;
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

template <typename T, int D, bool HALF>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvAppendArgs p) {
  constexpr int U = D / 8;
  const ttc_kv_append_t& a = p.a;
  const int u = threadIdx.x % U, e = 8 * u;
  const int64_t token = (int64_t)blockIdx.x * (256 / U) + threadIdx.x / U;
  if (token >= a.tokens) return;
  const int piece = blockIdx.y, heads = a.cache.heads;
  const bool value = piece >= p.q_pieces + heads;
  KvTurn t;
  bool lost = false;
  if (!value && a.rot) {
    const int64_t pos = a.positions[token];
    lost = (pos < 0 || pos >= a.table_rows) && e < a.rot;
    if (!lost) t = kv_turn<HALF>(a.table + pos * a.rot, a.rot, e, p.t_vec);
  }
  if (piece < p.q_pieces) {
    for (int i = 0; i < p.q_heads; ++i) {
      const int h = piece * p.q_heads + i;
      if (h >= a.heads_q) break;
      float y[8];
      const T* x = static_cast<const T*>(a.q) + token * a.q_token + h * a.q_head;
      kv_load_turned<T, HALF>(x, lost ? 0 : a.rot, e, p.q_vec, t, y);
      // in place the partners of a pair are read by two threads of one wavefront: all of its reads come before its writes
      __builtin_amdgcn_wave_barrier();
      if (lost) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = e + k < a.rot ? __builtin_nanf("") : y[k];
      }
      srv_st8(static_cast<T*>(a.q_out) + token * a.q_out_token + h * a.q_out_head + e, p.qo_vec, y);
    }
    return;
  }
  const int64_t slot = a.slots[token];
  const int page = a.cache.page, log_page = __builtin_ctz(page);
  if (slot < 0 || slot >= a.cache.pages * page) return;
  const int h = piece - p.q_pieces - (value ? heads : 0);
  float y[8];
  if (value) {
    srv_ld8(static_cast<const T*>(a.v) + token * a.v_token + h * a.v_head + e, p.v_vec, y);
  } else {
    kv_load_turned<T, HALF>(static_cast<const T*>(a.k) + token * a.k_token + h * a.k_head, lost ? 0 : a.rot, e, p.k_vec, t, y);
    if (lost) y[0] = __builtin_nanf("");
  }
  uint32_t exp;
  const uint32_t code = kv_quantise(y, exp);
  unsigned char* base = static_cast<unsigned char*>(a.cache.data) + ((slot >> log_page) * heads + h) * (int64_t)KvParts<D>::bytes(page);
  const KvPlace<D> at((int)(slot & (page - 1)), u, page);
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

// eight entries from their codes
__device__ __forceinline__ void kv_numbers(uint32_t code, uint32_t e, float (&x)[8]) {
  const float scale = e == 255 ? __builtin_nanf("") : e == 0 ? __uint_as_float(0x00400000u) : srv_scale(e);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = (code >> (4 * i)) & 15, m = c & 7;
    // magnitudes 0 .5 1 1.5 2 3 4 6: exponent and mantissa of a float32, apart from the first two
    const float v = m < 2 ? 0.5f * m : __uint_as_float(0x3f800000u + ((m - 2) << 22));
    x[i] = (c & 8 ? -v : v) * scale;
  }
}

template <typename T, int D>
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
  if (k) srv_st8(k + row, true, x);
  if (v) srv_st8(v + row, true, y);
}

}  // namespace ttc
