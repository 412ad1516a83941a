// kv_append_kernel, kv_read_kernel (ttc_kv_append, ttc_kv_read).
#include "ttc_kv.hpp"
#include "ttc_serve_launch.hpp"

namespace ttc {

static bool rows_of_16_bytes(const void* p, int64_t token, int64_t head, bool bf16) {
  return (uint64_t)p % 16 == 0 && (token | head) % (bf16 ? 8 : 4) == 0;
}

template <typename T, int D>
static void append(const KvAppendArgs& p, hipStream_t st) {
  constexpr int TOKENS = 256 / (D / 8);
  const dim3 grid((unsigned)((p.a.tokens + TOKENS - 1) / TOKENS), (unsigned)(p.q_pieces + 2 * p.a.cache.heads));
  if (p.a.layout == TTC_ROPE_HALF) hipLaunchKernelGGL((kv_append_kernel<T, D, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((kv_append_kernel<T, D, false>), grid, dim3(256), 0, st, p);
}

hipError_t launch_kv_append(const ttc_kv_append_t& a, hipStream_t st) {
  const bool bf16 = a.dtype == TTC_BF16;
  KvAppendArgs p;
  p.a = a;
  p.q_heads = 1;
  p.q_pieces = a.q ? a.heads_q : 0;
  p.k_vec = rows_of_16_bytes(a.k, a.k_token, a.k_head, bf16);
  p.v_vec = rows_of_16_bytes(a.v, a.v_token, a.v_head, bf16);
  p.q_vec = rows_of_16_bytes(a.q, a.q_token, a.q_head, bf16);
  p.qo_vec = rows_of_16_bytes(a.q_out, a.q_out_token, a.q_out_head, bf16);
  p.t_vec = (uint64_t)a.table % 16 == 0 && a.rot % 4 == 0;
  switch (a.cache.d) {
    case 64: bf16 ? append<unsigned short, 64>(p, st) : append<float, 64>(p, st); break;
    case 128: bf16 ? append<unsigned short, 128>(p, st) : append<float, 128>(p, st); break;
    case 256: bf16 ? append<unsigned short, 256>(p, st) : append<float, 256>(p, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T, int D>
static void read(const ttc_kv_cache_t& c, const int64_t* slots, int64_t n, void* k, void* v, hipStream_t st) {
  constexpr int TOKENS = 256 / (D / 8);
  hipLaunchKernelGGL((kv_read_kernel<T, D>), dim3((unsigned)((n + TOKENS - 1) / TOKENS), (unsigned)c.heads), dim3(256), 0, st, c, slots, n,
                     static_cast<T*>(k), static_cast<T*>(v));
}

hipError_t launch_kv_read(const ttc_kv_cache_t& c, const int64_t* slots, int64_t n, bool bf16, void* k, void* v, hipStream_t st) {
  switch (c.d) {
    case 64: bf16 ? read<unsigned short, 64>(c, slots, n, k, v, st) : read<float, 64>(c, slots, n, k, v, st); break;
    case 128: bf16 ? read<unsigned short, 128>(c, slots, n, k, v, st) : read<float, 128>(c, slots, n, k, v, st); break;
    case 256: bf16 ? read<unsigned short, 256>(c, slots, n, k, v, st) : read<float, 256>(c, slots, n, k, v, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace ttc
