// The norms, the gate and the residual scale around a block (ttc_residual_norm, ttc_residual_norm_backward).  Every row is read once and
// written once: the memory's rate bounds both.  A row is spread over LANES threads of a workgroup, eight features side by side to a thread and
// PIECES such eights, and stays in registers between the sums that its norms need.
#pragma once
#include "../../include/ttc_memory.h"
#include "ttc_serve.hpp"

namespace ttc {

struct NormArgs {
  ttc_residual_norm_t n;
  const void *gr, *gh;
  int64_t gr_token, gh_token;
  void *gy, *ggate, *gresidual;
  float* part[5];     // sums of one row of workgroups' threads each: post_gain, post_offset, residual_gain, pre_gain, pre_offset
  int32_t parts;      // rows of a part
  int32_t group;      // features of a group
  uint8_t vec;        // rows of 16-byte alignment: bits by NormRow
};
enum NormRow { ROW_Y, ROW_GATE, ROW_RESIDUAL, ROW_R, ROW_H };  // gr as r, gh as h

template <int LANES, int PIECES>
struct NormShape {
  static constexpr int THREADS = LANES < 256 ? 256 : LANES;
  static constexpr int ROWS = THREADS / LANES;  // of a workgroup
  static constexpr int WAVES = LANES / 64;      // of a row
};

// Sum over the LANES threads of a row, the same in all of them
template <int LANES>
__device__ __forceinline__ float norm_sum(float x, float* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
  if constexpr (LANES > 64) {
    __syncthreads();  // the last sum's readers are done
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x += lds[w];
  }
  return x;
}

// Sums over each group of the features that a thread's pieces belong to, in place.  Groups of 8, 16, .. 512 features lie within a wavefront;
// others meet in LDS.
template <int LANES, int PIECES>
__device__ __forceinline__ void norm_group_sums(float (&x)[PIECES], const NormArgs& a, float* lds, float* pieces) {
  if (a.n.groups == 1) {
    float whole = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) whole += x[i];
    whole = norm_sum<LANES>(whole, lds);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) x[i] = whole;
    return;
  }
  const int eights = a.group / 8;
  if (eights <= 64 && (eights & (eights - 1)) == 0) {
    for (int o = 1; o < eights; o <<= 1)
#pragma unroll
      for (int i = 0; i < PIECES; ++i) x[i] += __shfl_xor(x[i], o, 64);
    return;
  }
  const int at = threadIdx.x % LANES, row = threadIdx.x / LANES;
  float* mine = pieces + row * (LANES * PIECES);
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

// eight features from `e` on; those behind the last are 0
template <typename T>
__device__ __forceinline__ void norm_load(const T* row, int e, int features, bool vec, float (&x)[8]) {
  if (e + 8 <= features) {
    srv_ld8(row + e, vec, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = e + k < features ? srv_widen(row[e + k]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void norm_store(T* row, int e, int features, bool vec, const float (&x)[8]) {
  if (e + 8 <= features) {
    srv_stream8(row + e, vec, x);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (e + k < features) row[e + k] = srv_narrow<T>(x[k]);
  }
}
// of a vector of float32 numbers that every row reads, or `none` where there is no vector
__device__ __forceinline__ void norm_vector(const float* v, float none, int e, int features, float (&x)[8]) {
  if (!v) {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = none;
  } else {
    norm_load(v, e, features, (uint64_t)v % 16 == 0, x);
  }
}

// x -> (x - mean) / sqrt(mean square + eps) by groups; inverse: the factor.  The mean goes first, so that the squares are those of differences.
template <int LANES, int PIECES>
__device__ __forceinline__ void norm_unit(float (&x)[PIECES][8], int kind, float eps, const NormArgs& a, bool grouped, float (&inverse)[PIECES], float* lds,
                                          float* pieces) {
  const int at = threadIdx.x % LANES;
  const float n = (float)(grouped ? a.group : a.n.features);
  const auto sums = [&](float (&s)[PIECES]) {
    if (grouped) {
      norm_group_sums<LANES, PIECES>(s, a, lds, pieces);
    } else {
      float whole = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) whole += s[i];
      whole = norm_sum<LANES>(whole, lds);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) s[i] = whole;
    }
  };
  if (kind == TTC_NORM_LAYER) {
    float s[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      s[i] = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s[i] += x[i][k];
    }
    sums(s);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
#pragma unroll
      for (int k = 0; k < 8; ++k) x[i][k] = e + k < a.n.features ? x[i][k] - s[i] / n : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    inverse[i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) inverse[i] += x[i][k] * x[i][k];
  }
  sums(inverse);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    inverse[i] = 1.f / sqrtf(inverse[i] / n + eps);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[i][k] *= inverse[i];
  }
}

// A gradient with respect to unit entries becomes one with respect to the entries: inverse * (g - mean g [layer norm] - unit * mean (g * unit))
template <int LANES, int PIECES>
__device__ __forceinline__ void norm_unit_backward(float (&g)[PIECES][8], const float (&unit)[PIECES][8], const float (&inverse)[PIECES], int kind,
                                                   const NormArgs& a, bool grouped, float* lds, float* pieces) {
  const float n = (float)(grouped ? a.group : a.n.features);
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
  const auto sums = [&](float (&s)[PIECES]) {
    if (grouped) {
      norm_group_sums<LANES, PIECES>(s, a, lds, pieces);
    } else {
      float whole = 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) whole += s[i];
      whole = norm_sum<LANES>(whole, lds);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) s[i] = whole;
    }
  };
  sums(along);
  if (kind == TTC_NORM_LAYER) sums(mean);
#pragma unroll
  for (int i = 0; i < PIECES; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) g[i][k] = inverse[i] * (g[i][k] - (kind == TTC_NORM_LAYER ? mean[i] / n : 0.f) - unit[i][k] * (along[i] / n));
}

// act(x) and its derivative, from exp(-|x|), which never overflows; c = 1 - s comes without a cancellation.  Where a factor is 0 so is the
// product, of an infinite x too.
__device__ __forceinline__ void norm_act(int act, float x, float& y, float& slope) {
  if (act == TTC_GATE_IDENTITY) {
    y = x;
    slope = 1.f;
    return;
  }
  const float e = expf(-fabsf(x)), d = 1.f / (1.f + e), s = x < 0.f ? e * d : d, c = x < 0.f ? d : e * d;
  if (act == TTC_GATE_SIGMOID) {
    y = s;
    slope = s * c;
  } else {
    y = s == 0.f ? 0.f : x * s;
    slope = s == 0.f || c == 0.f ? s : s + x * s * c;
  }
}

template <typename T, int LANES, int PIECES>
__global__ void __launch_bounds__((NormShape<LANES, PIECES>::THREADS)) residual_norm_kernel(const NormArgs a) {
  typedef NormShape<LANES, PIECES> S;
  __shared__ float lds[16];
  __shared__ float pieces[S::THREADS * PIECES];
  const int at = threadIdx.x % LANES, c = a.n.features;
  const int64_t token = (int64_t)blockIdx.x * S::ROWS + threadIdx.x / LANES;
  const bool real = token < a.n.tokens;
  const int64_t t = real ? token : 0;  // (a wavefront behind the last row works on the first for nothing)
  const T* y = static_cast<const T*>(a.n.y) + t * a.n.y_token;
  const T* gate = a.n.gate ? static_cast<const T*>(a.n.gate) + t * a.n.gate_token : nullptr;
  const T* residual = a.n.residual ? static_cast<const T*>(a.n.residual) + t * a.n.residual_token : nullptr;
  float x[PIECES][8], g[PIECES][8], r[PIECES][8], inverse[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int e = (i * LANES + at) * 8;
    norm_load(y, e, c, a.vec >> ROW_Y & 1, x[i]);
    if (gate) norm_load(gate, e, c, a.vec >> ROW_GATE & 1, g[i]);
    if (residual) norm_load(residual, e, c, a.vec >> ROW_RESIDUAL & 1, r[i]);
  }
  if (a.n.post) norm_unit<LANES, PIECES>(x, a.n.post, a.n.post_eps, a, true, inverse, lds, pieces);
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int e = (i * LANES + at) * 8;
    float gain[8], offset[8], by[8];
    norm_vector(a.n.post ? a.n.post_gain : nullptr, 1.f, e, c, gain);
    norm_vector(a.n.post ? a.n.post_offset : nullptr, 0.f, e, c, offset);
    norm_vector(a.n.residual_gain, 1.f, e, c, by);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float z = x[i][k] * gain[k] + offset[k], act, slope;
      if (gate) {
        norm_act(a.n.act, g[i][k], act, slope);
        z *= act;
      }
      z *= a.n.scale * by[k];
      x[i][k] = e + k < c ? (residual ? r[i][k] + z : z) : 0.f;
    }
    if (real && a.n.r) norm_store(static_cast<T*>(a.n.r) + t * a.n.r_token, e, c, a.vec >> ROW_R & 1, x[i]);
  }
  if (!a.n.pre) return;
  norm_unit<LANES, PIECES>(x, a.n.pre, a.n.pre_eps, a, false, inverse, lds, pieces);
  if (!real) return;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int e = (i * LANES + at) * 8;
    float gain[8], offset[8];
    norm_vector(a.n.pre_gain, 1.f, e, c, gain);
    norm_vector(a.n.pre_offset, 0.f, e, c, offset);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[i][k] = x[i][k] * gain[k] + offset[k];
    norm_store(static_cast<T*>(a.n.h) + t * a.n.h_token, e, c, a.vec >> ROW_H & 1, x[i]);
  }
}

// Workgroups walk the rows with the sums over tokens in registers and leave one part of each sum for norm_parts_kernel: which rows make a
// part depends on the sizes alone.
template <typename T, int LANES, int PIECES>
__global__ void __launch_bounds__((NormShape<LANES, PIECES>::THREADS)) residual_norm_backward_kernel(const NormArgs a) {
  typedef NormShape<LANES, PIECES> S;
  __shared__ float lds[16];
  __shared__ float pieces[S::THREADS * PIECES];
  const int at = threadIdx.x % LANES, c = a.n.features, post = a.n.post, pre = a.n.pre;
  float sums[5][PIECES][8] = {};
  for (int64_t first = (int64_t)blockIdx.x * S::ROWS; first < a.n.tokens; first += (int64_t)gridDim.x * S::ROWS) {
    const int64_t token = first + threadIdx.x / LANES;
    const bool real = token < a.n.tokens;
    const int64_t t = real ? token : first;
    float x[PIECES][8], act[PIECES][8], slope[PIECES][8], total[PIECES][8], gh[PIECES][8], r[PIECES][8], inverse[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      norm_load(static_cast<const T*>(a.n.y) + t * a.n.y_token, e, c, a.vec >> ROW_Y & 1, x[i]);
      if (a.n.gate) norm_load(static_cast<const T*>(a.n.gate) + t * a.n.gate_token, e, c, a.vec >> ROW_GATE & 1, act[i]);
      if (a.gr) norm_load(static_cast<const T*>(a.gr) + t * a.gr_token, e, c, a.vec >> ROW_R & 1, total[i]);
      if (pre) {
        norm_load(static_cast<const T*>(a.gh) + t * a.gh_token, e, c, a.vec >> ROW_H & 1, gh[i]);
        if (a.n.residual) norm_load(static_cast<const T*>(a.n.residual) + t * a.n.residual_token, e, c, a.vec >> ROW_RESIDUAL & 1, r[i]);
      }
    }
    if (post) norm_unit<LANES, PIECES>(x, post, a.n.post_eps, a, true, inverse, lds, pieces);
    float z[PIECES][8], gain[PIECES][8];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      float offset[8], by[8];
      norm_vector(post ? a.n.post_gain : nullptr, 1.f, e, c, gain[i]);
      norm_vector(post ? a.n.post_offset : nullptr, 0.f, e, c, offset);
      norm_vector(a.n.residual_gain, 1.f, e, c, by);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        z[i][k] = x[i][k] * gain[i][k] + offset[k];
        if (a.n.gate) norm_act(a.n.act, act[i][k], act[i][k], slope[i][k]);
        else act[i][k] = 1.f;
        if (!a.gr) total[i][k] = 0.f;
        by[k] *= a.n.scale;
        if (pre) r[i][k] = e + k < c ? (a.n.residual ? r[i][k] : 0.f) + by[k] * act[i][k] * z[i][k] : 0.f;
      }
    }
    if (pre) {
      float unit_inverse[PIECES];
      norm_unit<LANES, PIECES>(r, pre, a.n.pre_eps, a, false, unit_inverse, lds, pieces);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int e = (i * LANES + at) * 8;
        float pre_gain[8];
        norm_vector(a.n.pre_gain, 1.f, e, c, pre_gain);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (real) {
            sums[3][i][k] += gh[i][k] * r[i][k];
            sums[4][i][k] += gh[i][k];
          }
          gh[i][k] *= pre_gain[k];
        }
      }
      norm_unit_backward<LANES, PIECES>(gh, r, unit_inverse, pre, a, false, lds, pieces);
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) total[i][k] += gh[i][k];
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int e = (i * LANES + at) * 8;
      if (real && a.gresidual) norm_store(static_cast<T*>(a.gresidual) + t * c, e, c, a.vec >> ROW_RESIDUAL & 1, total[i]);
      float by[8], ggate[8];
      norm_vector(a.n.residual_gain, 1.f, e, c, by);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float d = e + k < c ? total[i][k] * a.n.scale : 0.f;
        if (real) sums[2][i][k] += d * act[i][k] * z[i][k];
        if (a.n.gate) ggate[k] = d * by[k] * z[i][k] * slope[i][k];
        const float gz = d * by[k] * act[i][k];
        if (real) {
          sums[0][i][k] += gz * x[i][k];
          sums[1][i][k] += gz;
        }
        total[i][k] = gz * gain[i][k];
      }
      if (real && a.ggate) norm_store(static_cast<T*>(a.ggate) + t * c, e, c, a.vec >> ROW_GATE & 1, ggate);
    }
    if (post) norm_unit_backward<LANES, PIECES>(total, x, inverse, post, a, true, lds, pieces);
    if (real && a.gy)
#pragma unroll
      for (int i = 0; i < PIECES; ++i) norm_store(static_cast<T*>(a.gy) + t * c, (i * LANES + at) * 8, c, a.vec >> ROW_Y & 1, total[i]);
  }
  const int64_t part = (int64_t)blockIdx.x * S::ROWS + threadIdx.x / LANES;
#pragma unroll
  for (int v = 0; v < 5; ++v)
    if (a.part[v])
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int e = (i * LANES + at) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (e + k < c) a.part[v][part * c + e + k] = sums[v][i][k];
      }
}

struct NormParts {
  const float* part[5];
  float* out[5];
  int32_t parts, features, chunks;  // chunks: workgroups to a vector
};

// 64 features of one vector: four wavefronts a quarter of the parts each, added up in float64 (a feature may have 4096 parts)
static __global__ void __launch_bounds__(256) norm_parts_kernel(const NormParts a) {
  __shared__ double meet[4][64];
  const int v = blockIdx.x / a.chunks, e = blockIdx.x % a.chunks * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  double sum = 0.0;
  if (e < a.features)
    for (int p = wave; p < a.parts; p += 4) sum += a.part[v][(int64_t)p * a.features + e];
  meet[wave][threadIdx.x & 63] = sum;
  __syncthreads();
  if (wave == 0 && e < a.features) a.out[v][e] = (float)((meet[0][threadIdx.x] + meet[1][threadIdx.x]) + (meet[2][threadIdx.x] + meet[3][threadIdx.x]));
}

}  // namespace ttc
