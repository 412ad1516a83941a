// memory_chunk_kernel and memory_step_kernel for keys of up to TTC_D entries (ttc_linear_attention, ttc_linear_attention_backward).
#include "ttc_memory.hpp"
#include "ttc_memory_launch.hpp"

namespace ttc {

template <typename T, int NT>
static void chunks(const MemArgs& a, int what, uint32_t grid, hipStream_t st) {
  switch (what) {
    case MEM_STATES: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, NT, MEM_STATES>), dim3(grid), dim3(64 * MEM_WAVES), 0, st, a); break;
    case MEM_OUT: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, NT, MEM_OUT>), dim3(grid), dim3(64 * MEM_WAVES), 0, st, a); break;
    case MEM_OUT_DOTS: hipLaunchKernelGGL((memory_chunk_kernel<T, TTC_D, NT, MEM_OUT_DOTS>), dim3(grid), dim3(64 * MEM_WAVES), 0, st, a); break;
  }
}

template <>
hipError_t launch_memory_chunks<TTC_D>(const MemArgs& a, bool bf16, bool wide, int what, uint32_t grid, hipStream_t st) {
#if TTC_D <= 128
  if (wide) {
    if (bf16) chunks<unsigned short, 2>(a, what, grid, st);
    else chunks<float, 2>(a, what, grid, st);
    return hipGetLastError();
  }
#endif
  if (bf16) chunks<unsigned short, 1>(a, what, grid, st);
  else chunks<float, 1>(a, what, grid, st);
  return hipGetLastError();
}

template <>
hipError_t launch_memory_step<TTC_D>(const MemArgs& a, bool bf16, uint32_t grid, hipStream_t st) {
  if (bf16) hipLaunchKernelGGL((memory_step_kernel<unsigned short, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((memory_step_kernel<float, TTC_D>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace ttc
