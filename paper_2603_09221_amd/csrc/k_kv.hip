// kv_append_kernel, kv_read_kernel (ttc_kv_append, ttc_kv_read).
#include "ttc_kv.hpp"
#include "ttc_serve_launch.hpp"

namespace ttc {

static bool rows_of_16_bytes(const void* p, int64_t token, int64_t head, bool bf16) {
  return (uint64_t)p % 16 == 0 && (token | head) % (bf16 ? 8 : 4) == 0;
}

template <typename T, int D, int N>
static void append_many(KvAppendArgs& p, hipStream_t st) {
  constexpr int TOKENS = 256 / (D / 8);
  p.cache_workgroups = (uint32_t)((p.a.tokens + N * TOKENS - 1) / (N * TOKENS) * 2 * p.a.cache.heads);
  p.q_pieces = p.a.q ? (p.a.heads_q + N - 1) / N : 0;
  const dim3 grid(p.cache_workgroups + (unsigned)((p.a.tokens + TOKENS - 1) / TOKENS * p.q_pieces));
  if (p.a.layout == TTC_ROPE_HALF) hipLaunchKernelGGL((kv_append_kernel<T, D, true, N>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((kv_append_kernel<T, D, false, N>), grid, dim3(256), 0, st, p);
}

// A thread takes four query heads, which share the cosines it reads, or four tokens of a cache head, whose reads are under way together,
// once there are two workgroups to a compute unit that way.  One / four, us, 32 query and 8 cache heads of 128: 512 tokens 4.8 / 5.8, 1024
// 8.0 / 6.0, 2048 13.4 / 10.4, 16384 102 / 66; 16 and 16 heads of 64 in float32: 1024 tokens 4.5 / 5.7, 2048 7.7 / 7.5.
template <typename T, int D>
static void append(KvAppendArgs& p, int cus, hipStream_t st) {
  const int64_t heads = (p.a.q ? p.a.heads_q : 0) + 2ll * p.a.cache.heads;
  if (p.a.tokens * heads * (D / 8) >= 2ll * 256 * KV_MANY * cus) append_many<T, D, KV_MANY>(p, st);
  else append_many<T, D, 1>(p, st);
}

hipError_t launch_kv_append(const ttc_kv_append_t& a, int cus, hipStream_t st) {
  const bool bf16 = a.dtype == TTC_BF16;
  KvAppendArgs p;
  p.a = a;
  p.k_vec = rows_of_16_bytes(a.k, a.k_token, a.k_head, bf16);
  p.v_vec = rows_of_16_bytes(a.v, a.v_token, a.v_head, bf16);
  p.q_vec = rows_of_16_bytes(a.q, a.q_token, a.q_head, bf16);
  p.qo_vec = rows_of_16_bytes(a.q_out, a.q_out_token, a.q_out_head, bf16);
  p.t_vec = (uint64_t)a.table % 16 == 0 && a.rot % 4 == 0;
  switch (a.cache.d) {
    case 64: bf16 ? append<unsigned short, 64>(p, cus, st) : append<float, 64>(p, cus, st); break;
    case 128: bf16 ? append<unsigned short, 128>(p, cus, st) : append<float, 128>(p, cus, st); break;
    case 256: bf16 ? append<unsigned short, 256>(p, cus, st) : append<float, 256>(p, cus, st); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T, int D>
static void read(const ttc_kv_cache_t& c, const int64_t* slots, int64_t n, void* k, void* v, hipStream_t st) {
  constexpr int TOKENS = 256 / (D / 8);
  const dim3 grid((unsigned)((n + TOKENS - 1) / TOKENS), (unsigned)c.heads);
  // from 16 MiB of results on they are written past the caches: 16384 tokens of 8 heads of 128 take 16 us instead of 22
  if (2 * n * c.heads * D * (int64_t)sizeof(T) >= (16ll << 20))
    hipLaunchKernelGGL((kv_read_kernel<T, D, true>), grid, dim3(256), 0, st, c, slots, n, static_cast<T*>(k), static_cast<T*>(v));
  else
    hipLaunchKernelGGL((kv_read_kernel<T, D, false>), grid, dim3(256), 0, st, c, slots, n, static_cast<T*>(k), static_cast<T*>(v));
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
