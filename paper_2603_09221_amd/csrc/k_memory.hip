// memory_chunk_kernel and memory_step_kernel for keys of up to TTC_D entries (ttc_linear_attention, ttc_linear_attention_backward).
#include "ttc_memory.hpp"
#include "ttc_memory_launch.hpp"

namespace ttc {

template <typename T, int WAVES>
static void chunks(const MemTwo& a, int what, uint32_t grid, hipStream_t st) {
  switch (what) {
    case MEM_STATES: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, WAVES, MEM_STATES>), dim3(grid), dim3(64 * WAVES), 0, st, a); break;
    case MEM_OUT: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, WAVES, MEM_OUT>), dim3(grid), dim3(64 * WAVES), 0, st, a); break;
    case MEM_OUT_PAIRS: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, WAVES, MEM_OUT_PAIRS>), dim3(grid), dim3(64 * WAVES), 0, st, a); break;
    case MEM_OUT_DOTS: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, WAVES, MEM_OUT_DOTS>), dim3(grid), dim3(64 * WAVES), 0, st, a); break;
  }
}

template <>
hipError_t launch_memory_chunks<TTC_D>(const MemTwo& a, bool bf16, int columns, int what, uint32_t grid, hipStream_t st) {
  if (columns == 128) {
    if (bf16) chunks<unsigned short, 8>(a, what, grid, st);
#if TTC_D <= 128
    else chunks<float, 8>(a, what, grid, st);
#else
    else return hipErrorInvalidValue;  // (not in LDS)
#endif
  } else {
    if (bf16) chunks<unsigned short, 4>(a, what, grid, st);
    else chunks<float, 4>(a, what, grid, st);
  }
  return hipGetLastError();
}

template <>
hipError_t launch_memory_step<TTC_D>(const MemArgs& a, bool bf16, uint32_t grid, hipStream_t st) {
  if (bf16) hipLaunchKernelGGL((memory_step_kernel<unsigned short, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((memory_step_kernel<float, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ttc
