// memory_chunk_kernel and memory_step_kernel for keys of up to TTC_D entries (ttc_linear_attention, ttc_linear_attention_backward).
#include "ttc_memory.hpp"
#include "ttc_memory_launch.hpp"

namespace ttc {

template <typename T, int NT>
static void chunks(const MemArgs& a, bool states, uint32_t grid, hipStream_t st) {
  if (states) hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, NT, true>), dim3(grid), dim3(64 * MEM_WAVES), 0, st, a);
  else hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, NT, false>), dim3(grid), dim3(64 * MEM_WAVES), 0, st, a);
}

template <>
hipError_t launch_memory_chunks<TTC_D>(const MemArgs& a, bool bf16, bool wide, bool states, uint32_t grid, hipStream_t st) {
#if TTC_D <= 128
  if (wide) {
    if (bf16) chunks<unsigned short, 2>(a, states, grid, st);
    else chunks<float, 2>(a, states, grid, st);
    return hipGetLastError();
  }
#endif
  if (bf16) chunks<unsigned short, 1>(a, states, grid, st);
  else chunks<float, 1>(a, states, grid, st);
  return hipGetLastError();
}

template <>
hipError_t launch_memory_step<TTC_D>(const MemArgs& a, bool bf16, uint32_t grid, hipStream_t st) {
  if (bf16) hipLaunchKernelGGL((memory_step_kernel<unsigned short, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((memory_step_kernel<float, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ttc
