// Entry points of include/ttc_attention.h: argument checks and the launches.  The kernels live in k_rope.hip, k_kv.hip, k_place.hip, k_attention.hip.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <time.h>

#include <atomic>
#include <mutex>

#include "../../include/ttc_attention.h"
#include "ttc_serve_launch.hpp"

namespace ttc {

// compute units of the current device, asked once per device
int compute_units() {
  constexpr int MAX = 64;
  static std::once_flag once[MAX];
  static int count[MAX];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    dev = 0;
  }
  dev = dev < 0 || dev >= MAX ? 0 : dev;
  std::call_once(once[dev], [dev] {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
      (void)hipGetLastError();
      n = 256;  // MI355X
    }
    count[dev] = n;
  });
  return count[dev];
}

}  // namespace ttc

namespace {

using ttc::compute_units;

bool aligned(const void* p, uint64_t n) { return (uint64_t)p % n == 0; }
bool known_dtype(int32_t t) { return t == TTC_F32 || t == TTC_BF16; }
uint64_t bytes_of(int32_t t) { return t == TTC_BF16 ? 2 : 4; }

// 64 bits that what lies in a workspace has by chance only: a counter from a starting point of the process's own, mixed
uint64_t next_mark() {
  static std::atomic<uint64_t> calls{(uint64_t)time(nullptr) * 0x9e3779b97f4a7c15ull ^ (uint64_t)&calls ^ (uint64_t)clock()};
  uint64_t x = calls.fetch_add(0x9e3779b97f4a7c15ull, std::memory_order_relaxed);
  x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;
  x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
  x ^= x >> 31;
  return x ? x : 1;  // (a mark taken away is 0)
}

ttc_status_t check_rope(int32_t d, int32_t rot, int32_t layout, const int64_t* positions, const float* table, int64_t table_rows) {
  if (rot < 0 || rot > d || rot % 2 || (layout != TTC_ROPE_HALF && layout != TTC_ROPE_INTERLEAVED)) return TTC_ERR_INVALID_ARG;
  if (rot && (!positions || !table || table_rows < 1 || !aligned(positions, 8) || !aligned(table, 8))) return TTC_ERR_INVALID_ARG;
  return TTC_OK;
}

ttc_status_t check_cache(const ttc_kv_cache_t& c) {
  if (c.pages < 0 || c.heads < 1) return TTC_ERR_INVALID_ARG;
  if (!ttc_kv_page_bytes(c.d, c.page) || c.pages > (1ll << 40)) return TTC_ERR_UNSUPPORTED;
  if (c.pages && (!c.data || !aligned(c.data, 16))) return TTC_ERR_INVALID_ARG;
  return TTC_OK;
}

ttc_status_t run_rope(const ttc_rope_t* r, bool backward, void* hip_stream) {
  if (!r || r->tokens < 0 || r->heads < 1 || r->d < 1 || !known_dtype(r->dtype)) return TTC_ERR_INVALID_ARG;
  if (!r->tokens) return TTC_OK;
  if (const ttc_status_t s = check_rope(r->d, r->rot, r->layout, r->positions, r->table, r->table_rows); s != TTC_OK) return s;
  if (!r->x || !r->y || !aligned(r->x, bytes_of(r->dtype)) || !aligned(r->y, bytes_of(r->dtype))) return TTC_ERR_INVALID_ARG;
  if (r->x == r->y && (r->x_token != r->y_token || r->x_head != r->y_head)) return TTC_ERR_INVALID_ARG;
  if ((int64_t)r->heads * r->d > (1 << 26)) return TTC_ERR_UNSUPPORTED;
  return ttc::launch_rope(*r, backward, compute_units(), static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

// Checks what does not depend on tensors, and plans the call
ttc_status_t check_attention(const ttc_attention_t* a, ttc::AttentionArgs& p) {
  if (!a || a->sequences < 0 || a->tokens < 0 || !known_dtype(a->dtype) || a->max_q < 0 || a->max_kv < 0) return TTC_ERR_INVALID_ARG;
  if ((a->causal != 0 && a->causal != 1) || a->window < 0 || (a->window && !a->causal) || !isfinite(a->scale)) return TTC_ERR_INVALID_ARG;
  if (const ttc_status_t s = check_cache(a->cache); s != TTC_OK) return s;
  if (a->heads_q < 1 || a->heads_q % a->cache.heads) return TTC_ERR_INVALID_ARG;
  p.a = *a;
  return ttc::plan_attention(p, compute_units()) ? TTC_OK : TTC_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

ttc_status_t ttc_rope(const ttc_rope_t* rope, void* hip_stream) { return run_rope(rope, false, hip_stream); }

ttc_status_t ttc_rope_backward(const ttc_rope_t* rope, void* hip_stream) { return run_rope(rope, true, hip_stream); }

ttc_status_t ttc_rope_table(float* table, int64_t rows, int32_t pairs, const double* freqs, double scale, void* hip_stream) {
  if (rows < 0 || pairs < 0) return TTC_ERR_INVALID_ARG;
  if (!rows || !pairs) return TTC_OK;
  if (!table || !freqs || !aligned(table, 8) || !aligned(freqs, 8) || !isfinite(scale)) return TTC_ERR_INVALID_ARG;
  if (rows > (1ll << 40)) return TTC_ERR_UNSUPPORTED;
  return ttc::launch_rope_table(table, rows, pairs, freqs, scale, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

size_t ttc_kv_page_bytes(int32_t d, int32_t page) {
  if ((d != 64 && d != 128 && d != 256) || page < 16 || page > 256 || (page & (page - 1))) return 0;
  return (size_t)page * (d + d / 16);
}

ttc_status_t ttc_kv_append(const ttc_kv_append_t* a, void* hip_stream) {
  if (!a || a->tokens < 0 || !known_dtype(a->dtype)) return TTC_ERR_INVALID_ARG;
  if (const ttc_status_t s = check_cache(a->cache); s != TTC_OK) return s;
  if (!a->tokens) return TTC_OK;
  if (const ttc_status_t s = check_rope(a->cache.d, a->rot, a->layout, a->positions, a->table, a->table_rows); s != TTC_OK) return s;
  const uint64_t n = bytes_of(a->dtype);
  if (!a->k || !a->v || !a->slots || !aligned(a->k, n) || !aligned(a->v, n) || !aligned(a->slots, 8)) return TTC_ERR_INVALID_ARG;
  if (!a->q != !a->q_out || (a->q && (a->heads_q < 1 || !aligned(a->q, n) || !aligned(a->q_out, n)))) return TTC_ERR_INVALID_ARG;
  if (a->q && a->q == a->q_out && (a->q_token != a->q_out_token || a->q_head != a->q_out_head)) return TTC_ERR_INVALID_ARG;
  // a launch has fewer than 2^32 threads, one to eight entries
  if (a->tokens > (1 << 26) || (a->q ? (int64_t)a->heads_q : 0) + 2ll * a->cache.heads > 65535 ||
      (double)a->tokens * ((a->q ? a->heads_q : 0) + 2. * a->cache.heads) * a->cache.d >= 8. * 4e9) return TTC_ERR_UNSUPPORTED;
  return ttc::launch_kv_append(*a, compute_units(), static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

ttc_status_t ttc_kv_read(const ttc_kv_cache_t* c, const int64_t* slots, int64_t n, int32_t out_dtype, void* k_out, void* v_out, void* hip_stream) {
  if (!c || n < 0 || !known_dtype(out_dtype)) return TTC_ERR_INVALID_ARG;
  if (const ttc_status_t s = check_cache(*c); s != TTC_OK) return s;
  if (!n || (!k_out && !v_out)) return TTC_OK;
  if (!slots || !aligned(slots, 8) || !aligned(k_out, 16) || !aligned(v_out, 16)) return TTC_ERR_INVALID_ARG;
  if (n > (1 << 26) || c->heads > 65535) return TTC_ERR_UNSUPPORTED;  // (fewer than 2^32 threads along the tokens, 2^16 workgroups along the heads)
  return ttc::launch_kv_read(*c, slots, n, out_dtype == TTC_BF16, k_out, v_out, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

ttc_status_t ttc_kv_place(const ttc_kv_place_t* p, void* hip_stream) {
  if (!p || p->sequences < 0 || p->tokens < 0 || p->pages < 0 || p->width < 0) return TTC_ERR_INVALID_ARG;
  if (p->page < 1 || p->page > 65536 || p->sequences >= (1 << 30) || p->tokens >= (1 << 30) || p->pages > 0x7fffffffll) return TTC_ERR_UNSUPPORTED;
  if (!p->cu_q || !aligned(p->cu_q, 4)) return TTC_ERR_INVALID_ARG;
  if (p->sequences && (!p->past || !p->new_tokens || !p->kv_len || !aligned(p->past, 4) || !aligned(p->new_tokens, 4) || !aligned(p->kv_len, 4)))
    return TTC_ERR_INVALID_ARG;
  if (p->sequences && p->width && (!p->block_table || !aligned(p->block_table, 4) || p->table_stride < 0)) return TTC_ERR_INVALID_ARG;
  if (p->sequences > 1 && p->table_stride < p->width && p->free_pages) return TTC_ERR_INVALID_ARG;  // rows of the table would share pages
  if (p->tokens && (!p->positions || !p->slots || !aligned(p->positions, 8) || !aligned(p->slots, 8))) return TTC_ERR_INVALID_ARG;
  if (!aligned(p->sequence, 4) || !aligned(p->missing, 4)) return TTC_ERR_INVALID_ARG;
  if (p->free_pages && (!p->free_count || !p->free_count_out || p->free_capacity < 0 || p->free_capacity > 0x7fffffffll || !aligned(p->free_pages, 4) ||
                        !aligned(p->free_count, 4) || !aligned(p->free_count_out, 4))) return TTC_ERR_INVALID_ARG;
  return ttc::launch_kv_place(*p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

size_t ttc_attention_workspace_bytes(const ttc_attention_t* a) {
  ttc::AttentionArgs p;
  return check_attention(a, p) == TTC_OK ? ttc::attention_workspace(p) : 0;
}

ttc_status_t ttc_attention(const ttc_attention_t* a, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ttc::AttentionArgs p;
  if (const ttc_status_t s = check_attention(a, p); s != TTC_OK) return s;
  if (!a->sequences || !a->tokens || !a->max_q) return TTC_OK;
  const uint64_t n = bytes_of(a->dtype);
  if (!a->q || !a->out || !aligned(a->q, n) || !aligned(a->out, n) || !aligned(a->lse, 4) || a->q == a->out) return TTC_ERR_INVALID_ARG;
  if (!a->kv_len || !aligned(a->kv_len, 4) || !aligned(a->cu_q, 4)) return TTC_ERR_INVALID_ARG;
  if (a->max_kv && (!a->block_table || !aligned(a->block_table, 4) || a->table_stride < 0)) return TTC_ERR_INVALID_ARG;
  if (!a->cu_q && a->tokens != a->sequences) return TTC_ERR_INVALID_ARG;
  const uint64_t need = ttc::attention_workspace(p);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return TTC_ERR_WORKSPACE;
  ttc::place_workspace(p, workspace, next_mark());
  const bool bf16 = a->dtype == TTC_BF16;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipErrorInvalidValue;
  switch (a->cache.d) {
    case 64: e = ttc::launch_attention<64>(p, bf16, st); break;
    case 128: e = ttc::launch_attention<128>(p, bf16, st); break;
    case 256: e = ttc::launch_attention<256>(p, bf16, st); break;
  }
  return e == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

}  // extern "C"
