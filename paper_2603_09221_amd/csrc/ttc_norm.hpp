// The norms, the gate and the residual scale around a block (ttc_residual_norm, ttc_residual_norm_backward).  Every row is read once and
// written once: the memory's rate bounds both.  A row is spread over LANES threads of a workgroup, eight features side by side to a thread and
// PIECES such eights, and stays in registers between the sums that its norms need.  Workgroups walk the rows: what belongs to the features (gains,
// offsets, sums over tokens) stays in registers, and the next row is under way while one is worked on.
#pragma once
#include "../../include/ttc_memory.h"
#include "ttc_serve.hpp"

namespace ttc {

struct NormArgs {
  ttc_residual_norm_t n;
  const void *gr, *gh;
  int64_t gr_token, gh_token;
  void *gy, *ggate, *gresidual;
  float* part[5];     // sums over a workgroup's rows: post_gain, post_offset, residual_gain, pre_gain, pre_offset
  int32_t group;      // features of a group
};

// From 256 lanes on a workgroup has one row, and no more wavefronts than that has features for
template <int LANES, int PIECES>
struct NormShape {
  static constexpr int THREADS = LANES < 256 ? 256 : LANES;
  static constexpr int ROWS = THREADS / LANES;  // of a workgroup at once
  __device__ static __forceinline__ int row() { return LANES <= 256 ? threadIdx.x / LANES : 0; }  // (a number for all threads where there is one: addresses are, too)
  static int threads(int features) { return LANES < 256 || PIECES > 1 ? THREADS : (features + 511) / 512 * 64; }
};

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float norm_dpp(float x) {  // the number of another lane, 0 where there is none
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, true));
}

// Sum over a wavefront
__device__ __forceinline__ float norm_wave_sum(float x) {
  x += norm_dpp<0x111>(x);       // one to the right within 16 lanes, then two, four, eight
  x += norm_dpp<0x112>(x);
  x += norm_dpp<0x114>(x);
  x += norm_dpp<0x118>(x);
  x += norm_dpp<0x142, 0xa>(x);  // lane 15 to the next 16, lane 31 to the upper half
  x += norm_dpp<0x143, 0xc>(x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
// Sums over aligned sets of `lanes` lanes, a power of two
__device__ __forceinline__ float norm_lanes_sum(float x, int lanes) {
  if (lanes >= 2) x += norm_dpp<0xb1>(x);    // neighbours
  if (lanes >= 4) x += norm_dpp<0x4e>(x);    // pairs of them
  if (lanes >= 8) x += norm_dpp<0x141>(x);   // eight mirrored
  if (lanes >= 16) x += norm_dpp<0x140>(x);  // sixteen mirrored
  if (lanes >= 32) x += __shfl_xor(x, 16, 64);
  if (lanes >= 64) x += __shfl_xor(x, 32, 64);
  return x;
}

template <int LANES, int PIECES>
struct NormSums {
  typedef NormShape<LANES, PIECES> S;
  float (*meet)[16][2];  // two, in turn: a sum's writers need not wait for the readers of the last
  float* pieces;         // THREADS * PIECES
  int turn = 0;

  // N sums over the LANES threads of a row, the same in all of them
  template <int N>
  __device__ __forceinline__ void row(float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = norm_wave_sum(x[i]);
    if constexpr (LANES > 64) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) meet[turn][threadIdx.x >> 6][i] = x[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = 0.f;
      if constexpr (LANES == 1024) {  // one after the other: read ahead, 16 pairs take registers that are not there
#pragma unroll 2
        for (uint32_t w = 0; w < blockDim.x / 64; ++w)
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] += meet[turn][w][i];
      } else {
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w)
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] += meet[turn][threadIdx.x / LANES * (LANES / 64) + w][i];
      }
      turn ^= 1;
    }
  }

  // Sums over the group that each of a thread's pieces belongs to, in place.  Groups of 8, 16, .. 512 features lie within a wavefront; others
  // meet in LDS.
  __device__ __forceinline__ void group(float (&x)[PIECES], const NormArgs& a) {
    const int eights = a.group / 8;
    if (eights <= 64 && (eights & (eights - 1)) == 0) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) x[i] = norm_lanes_sum(x[i], eights);
      return;
    }
    const int at = threadIdx.x % LANES;
    float* mine = pieces + threadIdx.x / LANES * (LANES * PIECES);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) mine[i * LANES + at] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = i * LANES + at, first = e / eights * eights;
      float sum = 0.f;
      if (e * 8 < a.n.features)
        for (int k = 0; k < eights; ++k) sum += mine[first + k];
      x[i] = sum;
    }
  }

  // Sums of two numbers of every piece (the second only if `both`) over a row or over each group
  __device__ __forceinline__ void pair(float (&x)[PIECES], float (&y)[PIECES], bool both, const NormArgs& a, bool grouped) {
    if (grouped && a.n.groups > 1) {
      group(x, a);
      if (both) group(y, a);
      return;
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      s[0] += x[i];
      s[1] += y[i];
    }
    if (both) {
      row(s);
    } else {
      float t[1] = {s[0]};
      row(t);
      s[0] = t[0];
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      x[i] = s[0];
      y[i] = s[1];
    }
  }
};

// ---- rows ---------------------------------------------------------------------------------------------------------------

// Eight features as they lie in memory, in accesses of 16 bytes whatever the row's alignment: device memory takes them at that of a number
template <typename T> struct NormEight;
template <> struct NormEight<unsigned short> { srv_u16x8 x; };
template <> struct NormEight<float> { srv_floatx4 x[2]; };
typedef unsigned short norm_u16x8 __attribute__((ext_vector_type(8), aligned(2)));
typedef float norm_floatx4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void norm_fetch(const unsigned short* p, int e, int features, NormEight<unsigned short>& to) {
  if (e + 8 <= features) {
    to.x = __builtin_nontemporal_load(reinterpret_cast<const norm_u16x8*>(p + e));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) to.x[k] = e + k < features ? p[e + k] : 0;
  }
}
__device__ __forceinline__ void norm_fetch(const float* p, int e, int features, NormEight<float>& to) {
  if (e + 8 <= features) {
    to.x[0] = __builtin_nontemporal_load(reinterpret_cast<const norm_floatx4*>(p + e));
    to.x[1] = __builtin_nontemporal_load(reinterpret_cast<const norm_floatx4*>(p + e + 4));
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) to.x[k / 4][k % 4] = e + k < features ? p[e + k] : 0.f;
  }
}
__device__ __forceinline__ float norm_entry(const NormEight<unsigned short>& v, int k) { return srv_widen(v.x[k]); }
__device__ __forceinline__ float norm_entry(const NormEight<float>& v, int k) { return v.x[k / 4][k % 4]; }

__device__ __forceinline__ void norm_put(unsigned short* p, const float (&x)[8]) {
  srv_u16x8 v;
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = srv_narrow<unsigned short>(x[k]);
  __builtin_nontemporal_store(norm_u16x8(v), reinterpret_cast<norm_u16x8*>(p));
}
__device__ __forceinline__ void norm_put(float* p, const float (&x)[8]) {
  __builtin_nontemporal_store(norm_floatx4{x[0], x[1], x[2], x[3]}, reinterpret_cast<norm_floatx4*>(p));
  __builtin_nontemporal_store(norm_floatx4{x[4], x[5], x[6], x[7]}, reinterpret_cast<norm_floatx4*>(p + 4));
}
template <typename T>
__device__ __forceinline__ void norm_store(T* row, int e, int features, const float (&x)[8]) {
  if (e + 8 <= features) {
    norm_put(row + e, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (e + k < features) row[e + k] = srv_narrow<T>(x[k]);
  }
}
// of a vector of float32 numbers that every row reads, or `none` where there is no vector
__device__ __forceinline__ void norm_vector(const float* v, float none, int e, int features, float (&x)[8]) {
  if (v && e + 8 <= features) {
    srv_ld8(v + e, (uint64_t)v % 16 == 0, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = v && e + k < features ? v[e + k] : none;
  }
}

// x -> (x - mean) / sqrt(mean square + eps); inverse: the factor.  The mean goes first, so that the squares are those of differences.
template <int LANES, int PIECES>
__device__ __forceinline__ void norm_unit(float (&x)[PIECES][8], int kind, float eps, const NormArgs& a, bool grouped, float (&inverse)[PIECES],
                                          NormSums<LANES, PIECES>& sums) {
  const int at = threadIdx.x % LANES;
  const float share = 1.f / (float)(grouped ? a.group : a.n.features);
  float s[PIECES], none[PIECES] = {};
  if (kind == TTC_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      s[i] = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s[i] += x[i][k];
    }
    sums.pair(s, none, false, a, grouped);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[i][k] = e + k < a.n.features ? x[i][k] - s[i] * share : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    s[i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s[i] += x[i][k] * x[i][k];
  }
  sums.pair(s, none, false, a, grouped);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    inverse[i] = rsqrtf(s[i] * share + eps);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[i][k] *= inverse[i];
  }
}

// A gradient with respect to unit entries becomes one with respect to the entries: inverse * (g - mean g [layer norm] - unit * mean (g * unit))
template <int LANES, int PIECES>
__device__ __forceinline__ void norm_unit_backward(float (&g)[PIECES][8], const float (&unit)[PIECES][8], const float (&inverse)[PIECES], int kind,
                                                   const NormArgs& a, bool grouped, NormSums<LANES, PIECES>& sums) {
  const float share = 1.f / (float)(grouped ? a.group : a.n.features);
  float along[PIECES], mean[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    along[i] = mean[i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      along[i] += g[i][k] * unit[i][k];
      mean[i] += g[i][k];
    }
  }
  const bool layer = kind == TTC_NORM_LAYER;
  sums.pair(along, mean, layer, a, grouped);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const float l = along[i] * share;
    if (layer) {
      const int e = (i * LANES + threadIdx.x % LANES) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[i][k] -= e + k < a.n.features ? mean[i] * share : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) g[i][k] = inverse[i] * (g[i][k] - unit[i][k] * l);
  }
}

// act(x) and its derivative, from exp(-|x|), which never overflows; c = 1 - s comes without a cancellation.  Beyond 200 all is 0 or 1 in
// float32, and infinities there would meet zeros; NaN stays.  The exponential is a power of two of |x| / ln 2, whose rounding, |x| 2^-24, is made up for
// by 2^d = 1 + d ln 2; it is two steps off then, the reciprocal one.
__device__ __forceinline__ void norm_act(int act, float x, float& y, float& slope) {
  if (act == TTC_GATE_IDENTITY) {
    y = x;
    slope = 1.f;
    return;
  }
  const float low = x < -200.f ? -200.f : x, near = low > 200.f ? 200.f : low;
  constexpr double LOG2E = 1.44269504088896340736;
  constexpr float hi = (float)LOG2E, lo = (float)(LOG2E - hi);
  const float size = fabsf(near), power = size * -hi, rest = fmaf(size, -lo, fmaf(size, -hi, -power));
  const float rough = __builtin_amdgcn_exp2f(power), e = fmaf(rough, rest * 0.693147180559945309417f, rough);
  const float d = __builtin_amdgcn_rcpf(1.f + e), f = e * d;
  const float s = x < 0.f ? f : d, c = x < 0.f ? d : f;
  if (act == TTC_GATE_SIGMOID) {
    y = s;
    slope = s * c;
  } else {
    y = low * s;
    slope = s + near * s * c;
  }
}

// 16384 rows of 4096 bfloat16 with everything: 117 us, 5.7 TB/s.
template <typename T, int LANES, int PIECES>
__global__ void __launch_bounds__((NormShape<LANES, PIECES>::THREADS)) residual_norm_kernel(const NormArgs a) {
  typedef NormShape<LANES, PIECES> S;
  __shared__ float meet[2][16][2];
  __shared__ float pieces[S::THREADS * PIECES];
  if (LANES >= 256 && threadIdx.x < 64) (&meet[0][0][0])[threadIdx.x] = 0.f;  // those of wavefronts that are not there
  if (LANES >= 256) __syncthreads();
  NormSums<LANES, PIECES> sums = {meet, pieces};
  const int at = LANES <= 256 ? threadIdx.x % LANES : threadIdx.x, c = a.n.features;
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  // what belongs to the features, and the next row, as far as registers go: kept for all rows and under way beside one, else read anew
  constexpr bool KEEP = PIECES == 1;
  float post_gain[PIECES][8], post_offset[PIECES][8], by[PIECES][8], pre_gain[PIECES][8], pre_offset[PIECES][8];
  const auto vectors = [&](int i) {
    const int e = (i * LANES + at) * 8;
    norm_vector(a.n.post ? a.n.post_gain : nullptr, 1.f, e, c, post_gain[i]);
    norm_vector(a.n.post ? a.n.post_offset : nullptr, 0.f, e, c, post_offset[i]);
    norm_vector(a.n.residual_gain, 1.f, e, c, by[i]);
#pragma unroll
    for (int k = 0; k < 8; ++k) by[i][k] *= a.n.scale;
  };
  const auto vectors_after = [&](int i) {
    const int e = (i * LANES + at) * 8;
    norm_vector(a.n.pre_gain, 1.f, e, c, pre_gain[i]);
    norm_vector(a.n.pre_offset, 0.f, e, c, pre_offset[i]);
  };
  if (KEEP)
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      vectors(i);
      vectors_after(i);
    }
  NormEight<T> y[PIECES], gate[PIECES], residual[PIECES];
  const auto fetch = [&](int64_t t) {  // (behind the last row: the last once more, for nothing)
    t = t < a.n.tokens ? t : a.n.tokens - 1;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      norm_fetch(static_cast<const T*>(a.n.y) + t * a.n.y_token, e, c, y[i]);
      if (a.n.gate) norm_fetch(static_cast<const T*>(a.n.gate) + t * a.n.gate_token, e, c, gate[i]);
      if (a.n.residual) norm_fetch(static_cast<const T*>(a.n.residual) + t * a.n.residual_token, e, c, residual[i]);
    }
  };
  int64_t first = (int64_t)blockIdx.x * S::ROWS;
  if (KEEP) fetch(first + S::row());
  for (; first < a.n.tokens; first += step) {
    const int64_t t = first + S::row();
    const bool real = t < a.n.tokens;
    if (!KEEP) fetch(t);
    float x[PIECES][8], g[PIECES][8], r[PIECES][8], inverse[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[i][k] = norm_entry(y[i], k);
        if (a.n.gate) g[i][k] = norm_entry(gate[i], k);
        r[i][k] = a.n.residual ? norm_entry(residual[i], k) : 0.f;
      }
    if (KEEP && first + step < a.n.tokens) fetch(t + step);
    if (a.n.post) norm_unit<LANES, PIECES>(x, a.n.post, a.n.post_eps, a, true, inverse, sums);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      if (!KEEP) vectors(i);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float z = x[i][k] * post_gain[i][k] + post_offset[i][k], act, slope;
        if (a.n.gate) {
          norm_act(a.n.act, g[i][k], act, slope);
          z *= act;
        }
        x[i][k] = r[i][k] + by[i][k] * z;  // (0 behind the last feature: so are all its terms)
      }
      if (real && a.n.r) norm_store(static_cast<T*>(a.n.r) + t * a.n.r_token, e, c, x[i]);
    }
    if (!a.n.pre) continue;
    norm_unit<LANES, PIECES>(x, a.n.pre, a.n.pre_eps, a, false, inverse, sums);
    if (!real) continue;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      if (!KEEP) vectors_after(i);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[i][k] = x[i][k] * pre_gain[i][k] + pre_offset[i][k];
      norm_store(static_cast<T*>(a.n.h) + t * a.n.h_token, (i * LANES + at) * 8, c, x[i]);
    }
  }
}

// The sums over tokens stay in registers; a workgroup leaves one part of each for norm_parts_kernel, and which rows make a part depends on the
// sizes alone.  8192 rows of 4096 bfloat16 with everything: 130 us, 4.1 TB/s, on 8 wavefronts a compute unit, which is what 221 registers leave room for.
// OFFSETS: there are some, or their gradients are wanted
template <typename T, int LANES, int PIECES, bool OFFSETS>
__global__ void __launch_bounds__((NormShape<LANES, PIECES>::THREADS)) residual_norm_backward_kernel(const NormArgs a) {
  typedef NormShape<LANES, PIECES> S;
  constexpr int WIDTH = LANES * PIECES * 8;
  __shared__ float meet[2][16][2];
  __shared__ float pieces[S::ROWS > 1 ? S::ROWS * WIDTH : S::THREADS * PIECES];
  if (LANES >= 256 && threadIdx.x < 64) (&meet[0][0][0])[threadIdx.x] = 0.f;  // those of wavefronts that are not there
  if (LANES >= 256) __syncthreads();
  NormSums<LANES, PIECES> sums = {meet, pieces};
  int at = LANES <= 256 ? threadIdx.x % LANES : threadIdx.x;
  const int c = a.n.features, post = a.n.post, pre = a.n.pre;
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  float total_of[5][PIECES][8] = {};
  // As above.  With more than 512 threads a thread has 128 registers, and what belongs to the features would be spilled by all: 4096 rows of 8192 bfloat16 199 us
  // without offsets, 680 with all of it kept (415 with 512 threads of two eights each).  With two eights a gate is computed where it is needed, twice: 2048 rows
  // of 16384 603 us, 1005 with both its numbers kept.
  constexpr bool KEEP = LANES <= 512;
  float post_gain[PIECES][8], post_offset[PIECES][8], by[PIECES][8], pre_gain[PIECES][8];
  const auto vectors = [&](int i) {
    const int e = (i * LANES + at) * 8;
    norm_vector(post ? a.n.post_gain : nullptr, 1.f, e, c, post_gain[i]);
    norm_vector(OFFSETS && post ? a.n.post_offset : nullptr, 0.f, e, c, post_offset[i]);
    norm_vector(a.n.residual_gain, 1.f, e, c, by[i]);
  };
  const auto vectors_after = [&](int i) { norm_vector(a.n.pre_gain, 1.f, (i * LANES + at) * 8, c, pre_gain[i]); };
  if (KEEP)
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      vectors(i);
      vectors_after(i);
    }
  NormEight<T> y[PIECES], gate[PIECES], residual[PIECES], gr[PIECES], gh[PIECES];
  const auto fetch = [&](int64_t t) {  // (behind the last row: the last once more, for nothing)
    t = t < a.n.tokens ? t : a.n.tokens - 1;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      norm_fetch(static_cast<const T*>(a.n.y) + t * a.n.y_token, e, c, y[i]);
      if (a.n.gate) norm_fetch(static_cast<const T*>(a.n.gate) + t * a.n.gate_token, e, c, gate[i]);
      if (a.gr) norm_fetch(static_cast<const T*>(a.gr) + t * a.gr_token, e, c, gr[i]);
      if (pre) {
        norm_fetch(static_cast<const T*>(a.gh) + t * a.gh_token, e, c, gh[i]);
        if (a.n.residual) norm_fetch(static_cast<const T*>(a.n.residual) + t * a.n.residual_token, e, c, residual[i]);
      }
    }
  };
  int64_t first = (int64_t)blockIdx.x * S::ROWS;
  if (KEEP) fetch(first + S::row());
  for (; first < a.n.tokens; first += step) {
    const int64_t t = first + S::row();
    const bool real = t < a.n.tokens;
    if (!KEEP) {
      if (PIECES > 1) asm volatile("" : "+v"(at));  // places are found anew: kept, they would take registers that spill
      fetch(t);
    }
    float x[PIECES][8], act[PIECES][8], slope[PIECES][8], total[PIECES][8], g[PIECES][8], r[PIECES][8], inverse[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        x[i][k] = norm_entry(y[i], k);
        act[i][k] = a.n.gate ? norm_entry(gate[i], k) : 1.f;
        if (!KEEP) slope[i][k] = 0.f;  // (without a gate nobody reads it, but 43 registers are spilled instead of 27)
        total[i][k] = a.gr && real ? norm_entry(gr[i], k) : 0.f;
        if (pre) {
          g[i][k] = real ? norm_entry(gh[i], k) : 0.f;
          r[i][k] = a.n.residual ? norm_entry(residual[i], k) : 0.f;
        }
      }
    if (KEEP && first + step < a.n.tokens) fetch(t + step);
    if (post) norm_unit<LANES, PIECES>(x, post, a.n.post_eps, a, true, inverse, sums);
    const auto gates = [&](int i) {  // from the row as it came, where that is what is kept
      if (a.n.gate)
#pragma unroll
        for (int k = 0; k < 8; ++k) norm_act(a.n.act, PIECES == 1 ? act[i][k] : norm_entry(gate[i], k), act[i][k], slope[i][k]);
    };
    if constexpr (KEEP) {  // (the same, but for what the compiler makes of it: 338 us for 29484 rows of 1138, 422 through the lambda; wide rows the other way)
      if (a.n.gate)
#pragma unroll
        for (int k = 0; k < 8; ++k) norm_act(a.n.act, act[0][k], act[0][k], slope[0][k]);
    } else if (PIECES == 1) {
      gates(0);
    }
    if (pre) {
      float unit_inverse[PIECES];
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        if (!KEEP) vectors(i);
        if (PIECES > 1) gates(i);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float z = x[i][k] * post_gain[i][k] + post_offset[i][k];
          r[i][k] += a.n.scale * by[i][k] * (act[i][k] * z);
        }
      }
      norm_unit<LANES, PIECES>(r, pre, a.n.pre_eps, a, false, unit_inverse, sums);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        if (!KEEP) vectors_after(i);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          total_of[3][i][k] += g[i][k] * r[i][k];
          if (OFFSETS && a.part[4]) total_of[4][i][k] += g[i][k];
          g[i][k] *= pre_gain[i][k];
        }
      }
      norm_unit_backward<LANES, PIECES>(g, r, unit_inverse, pre, a, false, sums);
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) total[i][k] += g[i][k];
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      if (real && a.gresidual) norm_store(static_cast<T*>(a.gresidual) + t * c, e, c, total[i]);
      float ggate[8];
      if (!KEEP) vectors(i);
      if (PIECES > 1) gates(i);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float z = x[i][k] * post_gain[i][k] + post_offset[i][k];
        const float d = total[i][k] * a.n.scale;
        total_of[2][i][k] += d * act[i][k] * z;
        if (a.n.gate) ggate[k] = d * by[i][k] * z * slope[i][k];
        const float gz = d * by[i][k] * act[i][k];
        total_of[0][i][k] += gz * x[i][k];
        if (OFFSETS && a.part[1]) total_of[1][i][k] += gz;
        total[i][k] = gz * post_gain[i][k];
      }
      if (real && a.ggate) norm_store(static_cast<T*>(a.ggate) + t * c, e, c, ggate);
    }
    if (post) norm_unit_backward<LANES, PIECES>(total, x, inverse, post, a, true, sums);
    if (real && a.gy)
#pragma unroll
      for (int i = 0; i < PIECES; ++i) norm_store(static_cast<T*>(a.gy) + t * c, (i * LANES + at) * 8, c, total[i]);
  }
#pragma unroll
  for (int v = 0; v < 5; ++v)
    if ((OFFSETS || v % 3 != 1) && a.part[v]) {
      if constexpr (S::ROWS > 1) {
        float* mine = pieces + threadIdx.x / LANES * WIDTH;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) mine[(i * LANES + at) * 8 + k] = total_of[v][i][k];
        __syncthreads();
        for (int e = threadIdx.x; e < c; e += S::THREADS) {
          float sum = 0.f;
#pragma unroll
          for (int w = 0; w < S::ROWS; ++w) sum += pieces[w * WIDTH + e];
          a.part[v][(int64_t)blockIdx.x * c + e] = sum;
        }
      } else {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int e = (i * LANES + at) * 8;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (e + k < c) a.part[v][(int64_t)blockIdx.x * c + e + k] = total_of[v][i][k];
        }
      }
    }
}

struct NormParts {
  const float* part[5];
  float* out[5];
  int32_t parts, features, chunks;  // chunks: workgroups to a vector
};

constexpr int NORM_PARTS_WAVES = 16;

// 64 features of one vector, sixteen wavefronts a share of the parts each, added up in float64
static __global__ void __launch_bounds__(64 * NORM_PARTS_WAVES) norm_parts_kernel(const NormParts a) {
  __shared__ double meet[NORM_PARTS_WAVES][64];
  const int v = blockIdx.x / a.chunks, lane = threadIdx.x & 63, e = blockIdx.x % a.chunks * 64 + lane, wave = threadIdx.x >> 6;
  const float* from = a.part[v] + e;
  double sum = 0.0;
  if (e < a.features)
#pragma unroll 8
    for (int p = wave; p < a.parts; p += NORM_PARTS_WAVES) sum += from[(int64_t)p * a.features];
  meet[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && e < a.features) {
#pragma unroll
    for (int w = 1; w < NORM_PARTS_WAVES; ++w) sum += meet[w][lane];
    a.out[v][e] = (float)sum;
  }
}

}  // namespace ttc
