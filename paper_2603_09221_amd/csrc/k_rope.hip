// rope_kernel, rope_scalar_kernel, rope_table_kernel (ttc_rope, ttc_rope_backward, ttc_rope_table).
#include "ttc_rope.hpp"
#include "ttc_serve_launch.hpp"

namespace ttc {

// tokens of one launch: thread numbers stay below 2^31
static int64_t tokens_at_once(uint64_t threads_per_token) {
  const uint64_t n = 0x7fffff00ull / threads_per_token;
  return n < 1 ? 1 : (int64_t)n;
}

template <typename T, int VEC, bool HALF>
static void rope_vectors(const RopeArgs& a, bool many, dim3 grid, hipStream_t st) {
  if (many) hipLaunchKernelGGL((rope_kernel<T, VEC, HALF, ROPE_HEADS>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((rope_kernel<T, VEC, HALF, 1>), grid, dim3(256), 0, st, a);
}

hipError_t launch_rope(const ttc_rope_t& r, bool backward, int cus, hipStream_t st) {
  const bool bf16 = r.dtype == TTC_BF16, half = r.layout == TTC_ROPE_HALF;
  const int vec = bf16 ? 8 : 4;
  const uint64_t bits = (uint64_t)r.x | (uint64_t)r.y | (uint64_t)(r.rot ? r.table : nullptr);
  const int64_t steps = r.x_token | r.x_head | r.y_token | r.y_head;
  const bool vectors = bits % 16 == 0 && steps % vec == 0 && r.d % vec == 0 && (half ? r.rot / 2 : r.rot) % vec == 0;
  RopeArgs a;
  a.r = r;
  a.sign = backward ? -1.f : 1.f;
  const int rest = r.x == r.y ? 0 : r.d - r.rot;
  a.pairs = vectors ? (half ? r.rot / 2 : r.rot) / vec : r.rot / 2;
  a.units = a.pairs + (vectors ? rest / vec : rest);
  if (!a.units) return hipSuccess;
  // Four heads to a thread share the cosines they read, once every compute unit has a wavefront for each SIMD that way.  One / four, us,
  // 40 heads of 128: 64 tokens 2.7 / 3.5, 512 4.0 / 4.0, 2048 10.3 / 8.8, 16384 55.7 / 55.0.
  const bool many = vectors && (double)r.tokens * a.units * ((r.heads + ROPE_HEADS - 1) / ROPE_HEADS) >= 256. * cus;
  a.strides = many ? (r.heads + ROPE_HEADS - 1) / ROPE_HEADS : r.heads;
  const uint64_t per_token = (uint64_t)a.units * a.strides;
  if (per_token > 0x7fffff00ull) return hipErrorInvalidValue;
  const int64_t at_once = tokens_at_once(per_token);
  for (a.first = 0; a.first < r.tokens; a.first += at_once) {
    const int64_t n = r.tokens - a.first < at_once ? r.tokens - a.first : at_once;
    a.threads = (uint32_t)(n * per_token);
    const dim3 grid((a.threads + 255) / 256);
    if (vectors && bf16) half ? rope_vectors<unsigned short, 8, true>(a, many, grid, st) : rope_vectors<unsigned short, 8, false>(a, many, grid, st);
    else if (vectors) half ? rope_vectors<float, 4, true>(a, many, grid, st) : rope_vectors<float, 4, false>(a, many, grid, st);
    else if (bf16 && half) hipLaunchKernelGGL((rope_scalar_kernel<unsigned short, true>), grid, dim3(256), 0, st, a);
    else if (bf16) hipLaunchKernelGGL((rope_scalar_kernel<unsigned short, false>), grid, dim3(256), 0, st, a);
    else if (half) hipLaunchKernelGGL((rope_scalar_kernel<float, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((rope_scalar_kernel<float, false>), grid, dim3(256), 0, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_rope_table(float* table, int64_t rows, int32_t pairs, const double* freqs, double scale, hipStream_t st) {
  const int64_t at_once = tokens_at_once((uint64_t)pairs);
  for (int64_t first = 0; first < rows; first += at_once) {
    const int64_t n = rows - first < at_once ? rows - first : at_once;
    const uint32_t threads = (uint32_t)(n * pairs);
    hipLaunchKernelGGL(rope_table_kernel, dim3((threads + 255) / 256), dim3(256), 0, st, table, first, threads, (uint32_t)pairs, freqs, scale);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ttc
