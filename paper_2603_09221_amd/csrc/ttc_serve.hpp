// What the kernels of positions, cache and attention share (ttc_rope.hpp, ttc_kv.hpp, ttc_attention.hpp): element types, rows read
// and written in vectors where their alignment allows, and the addresses of the cache's four parts.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ttc_attention.h"

namespace ttc {

typedef float srv_floatx2 __attribute__((ext_vector_type(2)));
typedef float srv_floatx4 __attribute__((ext_vector_type(4)));
typedef unsigned int srv_uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned int srv_uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned short srv_u16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 srv_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 srv_bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float srv_widen(float x) { return x; }
__device__ __forceinline__ float srv_widen(unsigned short x) { return __uint_as_float(((uint32_t)x) << 16); }
template <typename T>
__device__ __forceinline__ T srv_narrow(float x);
template <>
__device__ __forceinline__ float srv_narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ unsigned short srv_narrow<unsigned short>(float x) {  // to nearest, ties to even
  return __builtin_bit_cast(unsigned short, static_cast<__bf16>(x));
}

// eight consecutive entries, in 16-byte accesses where `vec` says that the row allows it
__device__ __forceinline__ void srv_ld8(const float* p, bool vec, float (&x)[8]) {
  if (vec) {
    const srv_floatx4 a = *reinterpret_cast<const srv_floatx4*>(p), b = *reinterpret_cast<const srv_floatx4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
  }
}
__device__ __forceinline__ void srv_ld8(const unsigned short* p, bool vec, float (&x)[8]) {
  if (vec) {
    const srv_u16x8 a = *reinterpret_cast<const srv_u16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = srv_widen(a[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = srv_widen(p[i]);
  }
}
__device__ __forceinline__ srv_bf16x8 srv_ld8_bf16(const unsigned short* p, bool vec) {
  if (vec) return *reinterpret_cast<const srv_bf16x8*>(p);
  srv_u16x8 x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = p[i];
  return __builtin_bit_cast(srv_bf16x8, x);
}
__device__ __forceinline__ void srv_st8(float* p, bool vec, const float (&x)[8]) {
  if (vec) {
    *reinterpret_cast<srv_floatx4*>(p) = srv_floatx4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<srv_floatx4*>(p + 4) = srv_floatx4{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i];
  }
}
__device__ __forceinline__ void srv_st8(unsigned short* p, bool vec, const float (&x)[8]) {
  if (vec) {
    srv_u16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = srv_narrow<unsigned short>(x[i]);
    *reinterpret_cast<srv_u16x8*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = srv_narrow<unsigned short>(x[i]);
  }
}

// 4, 8 or 16 consecutive entries
template <typename T, int N>
__device__ __forceinline__ void srv_st(T* p, bool vec, const float (&x)[N]) {
  if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8) srv_st8(p + i, vec, reinterpret_cast<const float(&)[8]>(x[i]));
  } else {
    typedef T four_t __attribute__((ext_vector_type(4)));
    static_assert(N == 4);
    const four_t v = {srv_narrow<T>(x[0]), srv_narrow<T>(x[1]), srv_narrow<T>(x[2]), srv_narrow<T>(x[3])};
    if (vec) {
      *reinterpret_cast<four_t*>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = v[i];
    }
  }
}

// eight entries of a large result, past the caches' replacement
__device__ __forceinline__ void srv_stream8(float* p, bool vec, const float (&x)[8]) {
  if (vec) {
    __builtin_nontemporal_store(srv_floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<srv_floatx4*>(p));
    __builtin_nontemporal_store(srv_floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<srv_floatx4*>(p + 4));
  } else {
    srv_st8(p, false, x);
  }
}
__device__ __forceinline__ void srv_stream8(unsigned short* p, bool vec, const float (&x)[8]) {
  if (vec) {
    srv_u16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = srv_narrow<unsigned short>(x[i]);
    __builtin_nontemporal_store(v, reinterpret_cast<srv_u16x8*>(p));
  } else {
    srv_st8(p, false, x);
  }
}

// Two entries of a pair turned by (cos, sin): each product and the sum rounded on its own, so that the key that the cache takes is
// the same number, to the last bit, as the rotation gives by itself (a contracted multiply-add would round differently, and
// entries that lie between two codes would go the other way).
__device__ __forceinline__ void srv_turn(float a, float b, float c, float s, float& ya, float& yb) {
#pragma clang fp contract(off)
  const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
  ya = ac - bs;
  yb = bc + as;
}

// The four parts of one head of one page, in bytes from its start (include/ttc_attention.h)
template <int D>
struct KvParts {
  static constexpr int TOKEN = D / 2;          // codes of a token's keys
  static constexpr int LANE = D / 32;          // codes of a token's values that one of 16 lanes holds
  static constexpr int BLOCKS = D / 32;        // exponents of a token
  __host__ __device__ static constexpr int values(int page) { return page * TOKEN; }
  __host__ __device__ static constexpr int key_exps(int page) { return 2 * page * TOKEN; }
  __host__ __device__ static constexpr int value_exps(int page) { return 2 * page * TOKEN + page * BLOCKS; }
  __host__ __device__ static constexpr int bytes(int page) { return 2 * page * (TOKEN + BLOCKS); }
};

// an exponent byte as the float32 that the conversion instructions take for a scale (they read its exponent alone)
__device__ __forceinline__ float srv_scale(uint32_t e) { return __uint_as_float(e << 23); }
// the same of any byte: above 252, with which some codes would be infinite, a block is NaN
constexpr uint32_t KV_LARGEST = 252;
__device__ __forceinline__ float srv_scale_or_nan(uint32_t e) { return srv_scale(e > KV_LARGEST ? 255u : e); }

}  // namespace ttc
