// Host-side interface between the entry points of include/ttc_attention.h (ttc_api_attention.hip) and their kernels.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/ttc_attention.h"
#include "ttc_attention_plan.hpp"

namespace ttc {

hipError_t launch_rope(const ttc_rope_t& r, bool backward, int cus, hipStream_t st);
hipError_t launch_rope_table(float* table, int64_t rows, int32_t pairs, const double* freqs, double scale, hipStream_t st);
hipError_t launch_kv_append(const ttc_kv_append_t& a, int cus, hipStream_t st);
hipError_t launch_kv_read(const ttc_kv_cache_t& c, const int64_t* slots, int64_t n, bool bf16, void* k, void* v, hipStream_t st);
template <int D> hipError_t launch_attention(const AttentionArgs& a, bool bf16, hipStream_t st);

}  // namespace ttc
