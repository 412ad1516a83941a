// attention_kernel, attention_prompt_kernel (ttc_attention), for heads of TTC_D entries.
#include "ttc_attention_prompt.hpp"
#include "ttc_serve_launch.hpp"

namespace ttc {

template <typename T>
static hipError_t launch(const AttentionArgs& p, hipStream_t st) {
  if constexpr (prompt_kernel(sizeof(T) == 2, TTC_D)) {
    if (p.prompt) {
      hipLaunchKernelGGL((attention_prompt_kernel<T, TTC_D>), dim3((unsigned)p.workgroups), dim3(64 * PROMPT_WAVES), 0, st, p);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((attention_kernel<T, TTC_D>), dim3((unsigned)p.workgroups), dim3(64 * ATT_WAVES), 0, st, p);
  return hipGetLastError();
}

template <>
hipError_t launch_attention<TTC_D>(const AttentionArgs& p, bool bf16, hipStream_t st) {
  return bf16 ? launch<unsigned short>(p, st) : launch<float>(p, st);
}

}  // namespace ttc
