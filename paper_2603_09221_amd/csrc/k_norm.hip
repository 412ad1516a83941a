// residual_norm_kernel, residual_norm_backward_kernel, norm_parts_kernel (ttc_residual_norm, ttc_residual_norm_backward).
#include "ttc_memory_launch.hpp"
#include "ttc_norm.hpp"

namespace ttc {

// Threads of a compute unit: forward all that fit (16384 rows of 4096 bfloat16: 117 us; 120 with 2048, 123 with 1024); backward those that their registers
// leave room for at once, as every workgroup leaves a part of each sum (8192 rows of 4096: 130 us; 141 with 1024, 162 with 2048).
constexpr int NORM_THREADS = 4096, NORM_THREADS_BACKWARD = 512;

// A thread to every eight features as far as a workgroup goes: more eights to a thread take registers that the wavefronts in flight lack (two: 188 us
// forward where one takes 117, 301 us backward where one takes 130)
template <typename F>
static void norm_shape(int features, F&& f) {
  if (features <= 512) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else if (features <= 1024) f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  else if (features <= 2048) f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  else if (features <= 4096) f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  else if (features <= 8192) f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  else f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
}

hipError_t launch_residual_norm(const ttc_residual_norm_t& n, int cus, hipStream_t st) {
  NormArgs a = {};
  a.n = n;
  a.group = n.features / n.groups;
  norm_shape(n.features, [&](auto lanes, auto pieces) {
    typedef NormShape<decltype(lanes)::value, decltype(pieces)::value> S;
    const int threads = S::threads(n.features);
    const int64_t rows = (n.tokens + S::ROWS - 1) / S::ROWS, most = (int64_t)cus * (NORM_THREADS / threads);
    const dim3 grid((uint32_t)(rows < most ? rows : most));
    if (n.dtype == TTC_BF16) hipLaunchKernelGGL((residual_norm_kernel<unsigned short, lanes(), pieces()>), grid, dim3(threads), 0, st, a);
    else hipLaunchKernelGGL((residual_norm_kernel<float, lanes(), pieces()>), grid, dim3(threads), 0, st, a);
  });
  return hipGetLastError();
}

// Workgroups of the backward pass, each of which leaves a part of every sum
static int norm_grid(const ttc_residual_norm_t& n, int cus) {
  int grid = 0;
  norm_shape(n.features, [&](auto lanes, auto pieces) {
    typedef NormShape<decltype(lanes)::value, decltype(pieces)::value> S;
    const int64_t rows = (n.tokens + S::ROWS - 1) / S::ROWS, each = NORM_THREADS_BACKWARD / S::threads(n.features), most = cus * (each ? each : 1);
    grid = (int)(rows < most ? rows : most);
  });
  return grid;
}

static void norm_wanted(const ttc_residual_norm_backward_t& b, float* (&out)[5]) {
  out[0] = b.gpost_gain;
  out[1] = b.gpost_offset;
  out[2] = b.gresidual_gain;
  out[3] = b.gpre_gain;
  out[4] = b.gpre_offset;
}

uint64_t norm_backward_workspace(const ttc_residual_norm_backward_t& b, int cus) {
  int vectors = 0;
  float* out[5];
  norm_wanted(b, out);
  for (float* v : out) vectors += v != nullptr;
  return (uint64_t)vectors * norm_grid(b.forward, cus) * b.forward.features * 4;
}

hipError_t launch_residual_norm_backward(const ttc_residual_norm_backward_t& b, int cus, void* workspace, hipStream_t st) {
  const ttc_residual_norm_t& n = b.forward;
  NormArgs a = {};
  a.n = n;
  a.group = n.features / n.groups;
  a.gr = b.gr; a.gh = b.gh; a.gr_token = b.gr_token; a.gh_token = b.gh_token;
  a.gy = b.gy; a.ggate = b.ggate; a.gresidual = b.gresidual;
  const int grid = norm_grid(n, cus);
  NormParts sum = {};
  float* out[5];
  norm_wanted(b, out);
  float* at = static_cast<float*>(workspace);
  int vectors = 0;
  for (int v = 0; v < 5; ++v)
    if (out[v]) {
      a.part[v] = at;
      sum.part[vectors] = at;
      sum.out[vectors++] = out[v];
      at += (int64_t)grid * n.features;
    }
  sum.parts = grid;
  sum.features = n.features;
  sum.chunks = (n.features + 63) / 64;
  if (grid) norm_shape(n.features, [&](auto lanes, auto pieces) {
    typedef NormShape<decltype(lanes)::value, decltype(pieces)::value> S;
    constexpr bool wide = lanes() > 512;  // where registers are short
    const auto run = [&](auto type, auto offsets) {
      hipLaunchKernelGGL((residual_norm_backward_kernel<decltype(type), lanes(), pieces(), decltype(offsets)::value>), dim3(grid), dim3(S::threads(n.features)), 0, st, a);
    };
    const bool any = n.post_offset || a.part[1] || a.part[4];
    if (n.dtype == TTC_BF16) any || !wide ? run((unsigned short)0, std::true_type{}) : run((unsigned short)0, std::integral_constant<bool, !wide>{});
    else any || !wide ? run(0.f, std::true_type{}) : run(0.f, std::integral_constant<bool, !wide>{});
  });
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (vectors) hipLaunchKernelGGL(norm_parts_kernel, dim3(vectors * sum.chunks), dim3(64 * NORM_PARTS_WAVES), 0, st, sum);
  return hipGetLastError();
}

}  // namespace ttc
