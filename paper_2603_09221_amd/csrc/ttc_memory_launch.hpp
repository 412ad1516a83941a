// Host-side interface between the entry points of include/ttc_memory.h (ttc_api_memory.hip) and their kernels.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ttc_memory.h"

namespace ttc {

uint64_t linear_attention_workspace(const ttc_linear_attention_t& a, int cus);
hipError_t launch_linear_attention(const ttc_linear_attention_t& a, int cus, void* workspace, hipStream_t st);
uint64_t linear_attention_backward_workspace(const ttc_linear_attention_backward_t& b, int cus);
hipError_t launch_linear_attention_backward(const ttc_linear_attention_backward_t& b, int cus, void* workspace, hipStream_t st);

hipError_t launch_residual_norm(const ttc_residual_norm_t& n, int cus, hipStream_t st);
uint64_t norm_backward_workspace(const ttc_residual_norm_backward_t& b, int cus);
hipError_t launch_residual_norm_backward(const ttc_residual_norm_backward_t& b, int cus, void* workspace, hipStream_t st);

// rows of x and w of up to D entries; columns of a workgroup (64 or 128); what: a MemWhat
struct MemArgs;
struct MemTwo;
template <int D> hipError_t launch_memory_chunks(const MemTwo& a, bool bf16, int columns, int what, uint32_t grid, hipStream_t st);
template <int D> hipError_t launch_memory_step(const MemArgs& a, bool bf16, uint32_t grid, hipStream_t st);

}  // namespace ttc
