// place_sequences_kernel, place_tokens_kernel (ttc_kv_place).
#include "ttc_place.hpp"
#include "ttc_serve_launch.hpp"

namespace ttc {

hipError_t launch_kv_place(const ttc_kv_place_t& p, hipStream_t st) {
  const bool alone = p.tokens <= PLACE_ALONE;
  hipLaunchKernelGGL(place_sequences_kernel, dim3(1), dim3(PLACE_THREADS), 0, st, p, alone);
  if (!alone) {
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const int64_t each = 256 * PLACE_TOKENS;
    hipLaunchKernelGGL(place_tokens_kernel, dim3((uint32_t)((p.tokens + each - 1) / each)), dim3(256), 0, st, p);
  }
  return hipGetLastError();
}

}  // namespace ttc
