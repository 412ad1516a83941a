// Rotary positions (ttc_rope, ttc_rope_backward, ttc_rope_table).  Every entry is read once and written once: the memory's rate bounds
// it.  A thread owns 16 bytes of a head and of their partners, and walks several heads of one token with the cosines it has read once.
#pragma once
#include "ttc_serve.hpp"

namespace ttc {

struct RopeArgs {
  ttc_rope_t r;
  int64_t first;           // token of the launch's first thread
  uint32_t threads;        // of this launch
  uint32_t units, pairs;   // pieces of a head: those of pairs, then those copied
  uint32_t strides;        // a thread takes heads hc, hc + strides, ..
  float sign;              // of the sines: -1 for the transposed rotation
};

constexpr int ROPE_HEADS = 4;  // heads that a thread takes where there is enough work for it

// HEADS heads to a thread, all loads under way before the first is used.  What is read is read once, past the caches' replacement: 16384 tokens
// of 40 heads of 128 in 55 us instead of 66 (340 MB, 6.2 TB/s; with the results written that way too 57).
template <typename T, int VEC, bool HALF, int HEADS>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
  const uint32_t t = blockIdx.x * 256u + threadIdx.x;
  if (t >= a.threads) return;
  const uint32_t u = t % a.units, r = t / a.units, hc = r % a.strides;
  const int64_t token = a.first + r / a.strides;
  const T* x = static_cast<const T*>(a.r.x) + token * a.r.x_token;
  T* y = static_cast<T*>(a.r.y) + token * a.r.y_token;
  typedef T vec_t __attribute__((ext_vector_type(VEC)));
  const int half = a.r.rot / 2;
  if (u >= a.pairs) {  // entries behind the rotated ones
    const int e = a.r.rot + (int)(u - a.pairs) * VEC;
    vec_t v[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const uint32_t h = hc + i * a.strides;
      if (h < (uint32_t)a.r.heads) v[i] = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(x + h * a.r.x_head + e));
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const uint32_t h = hc + i * a.strides;
      if (h < (uint32_t)a.r.heads) *reinterpret_cast<vec_t*>(y + h * a.r.y_head + e) = v[i];
    }
    return;
  }
  constexpr int N = HALF ? VEC : VEC / 2;  // pairs of this thread in one head
  vec_t v[HEADS], w[HALF ? HEADS : 1];
  const int e = (int)u * VEC;
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const uint32_t h = hc + i * a.strides;
    if (h < (uint32_t)a.r.heads) {
      v[i] = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(x + h * a.r.x_head + e));
      if constexpr (HALF) w[i] = __builtin_nontemporal_load(reinterpret_cast<const vec_t*>(x + h * a.r.x_head + half + e));
    }
  }
  float c[N], s[N];
  const int64_t pos = a.r.positions[token];
  if (pos >= 0 && pos < a.r.table_rows) {
    const srv_floatx4* cs = reinterpret_cast<const srv_floatx4*>(a.r.table + (pos * half + (int)u * N) * 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const srv_floatx4 q = cs[i];
      c[2 * i] = q[0]; s[2 * i] = a.sign * q[1]; c[2 * i + 1] = q[2]; s[2 * i + 1] = a.sign * q[3];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = s[i] = __builtin_nanf("");
  }
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const uint32_t h = hc + i * a.strides;
    if (h >= (uint32_t)a.r.heads) break;
    vec_t p, q;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float ya, yb;
      if constexpr (HALF) {
        srv_turn(srv_widen(v[i][k]), srv_widen(w[i][k]), c[k], s[k], ya, yb);
        p[k] = srv_narrow<T>(ya);
        q[k] = srv_narrow<T>(yb);
      } else {
        srv_turn(srv_widen(v[i][2 * k]), srv_widen(v[i][2 * k + 1]), c[k], s[k], ya, yb);
        p[2 * k] = srv_narrow<T>(ya);
        p[2 * k + 1] = srv_narrow<T>(yb);
      }
    }
    *reinterpret_cast<vec_t*>(y + h * a.r.y_head + e) = p;
    if constexpr (HALF) *reinterpret_cast<vec_t*>(y + h * a.r.y_head + half + e) = q;
  }
}

// rows whose size, stride or address does not allow vectors: a thread owns one pair, or one copied entry
template <typename T, bool HALF>
__global__ void __launch_bounds__(256) rope_scalar_kernel(const RopeArgs a) {
  const uint32_t t = blockIdx.x * 256u + threadIdx.x;
  if (t >= a.threads) return;
  const uint32_t u = t % a.units, r = t / a.units, h = r % a.strides;
  const int64_t token = a.first + r / a.strides;
  const T* x = static_cast<const T*>(a.r.x) + token * a.r.x_token + h * a.r.x_head;
  T* y = static_cast<T*>(a.r.y) + token * a.r.y_token + h * a.r.y_head;
  if (u >= a.pairs) {
    const int e = a.r.rot + (int)(u - a.pairs);
    y[e] = x[e];
    return;
  }
  const int half = a.r.rot / 2, e0 = HALF ? (int)u : 2 * (int)u, e1 = HALF ? (int)u + half : 2 * (int)u + 1;
  const int64_t pos = a.r.positions[token];
  float c = __builtin_nanf(""), s = c;
  if (pos >= 0 && pos < a.r.table_rows) {
    const float* cs = a.r.table + (pos * half + (int)u) * 2;
    c = cs[0];
    s = a.sign * cs[1];
  }
  float ya, yb;
  srv_turn(srv_widen(x[e0]), srv_widen(x[e1]), c, s, ya, yb);
  y[e0] = srv_narrow<T>(ya);
  y[e1] = srv_narrow<T>(yb);
}

// The angle in float64: at position 10^6 and frequency 1 float32 would leave the angle itself 0.03 off.
static __global__ void __launch_bounds__(256) rope_table_kernel(float* table, int64_t first, uint32_t threads, uint32_t pairs,
                                                                const double* freqs, double scale) {
  const uint32_t t = blockIdx.x * 256u + threadIdx.x;
  if (t >= threads) return;
  const uint32_t i = t % pairs;
  const int64_t p = first + t / pairs;
  double s, c;
  sincos((double)p * freqs[i], &s, &c);
  *reinterpret_cast<srv_floatx2*>(table + (p * pairs + i) * 2) = srv_floatx2{(float)(scale * c), (float)(scale * s)};
}

}  // namespace ttc
