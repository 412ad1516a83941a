// Entry points of include/ttc_memory.h: argument checks and the launches.  The kernels live in k_memory.hip, k_memory_host.hip, k_norm.hip.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ttc_memory_launch.hpp"
#include "ttc_serve_launch.hpp"

namespace {

bool aligned(const void* p, uint64_t n) { return (uint64_t)p % n == 0; }
bool known_dtype(int32_t t) { return t == TTC_F32 || t == TTC_BF16; }
uint64_t bytes_of(int32_t t) { return t == TTC_BF16 ? 2 : 4; }

// Memory that a call reads or writes: `count` rows of `width` bytes, `step` bytes apart
struct Rows {
  uint64_t at;
  int64_t count, step;
  uint64_t width;
};

Rows whole(const void* p, uint64_t bytes) { return {(uint64_t)p, p && bytes ? 1 : 0, 0, bytes}; }
// of tokens, with the space between their heads; strides in entries of `size` bytes
Rows rows_of(const void* p, int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t entries, uint64_t size) {
  uint64_t at = (uint64_t)p;
  if (head < 0) at += (heads - 1) * head * (int64_t)size;
  if (token < 0 && tokens > 1) at += (tokens - 1) * token * (int64_t)size;
  return {at, p ? tokens : 0, (token < 0 ? -token : token) * (int64_t)size, ((heads - 1) * (head < 0 ? -head : head) + entries) * size};
}
// Whether `one` block of memory and rows have a byte in common
bool meet(const Rows& one, const Rows& r) {
  if (!one.count || r.count < 1) return false;
  const uint64_t end = one.at + one.width;
  if (r.count == 1 || (uint64_t)r.step <= r.width) return one.at < r.at + (r.count - 1) * r.step + r.width && r.at < end;
  if (r.at >= end) return false;
  const uint64_t behind = r.at + r.width;  // of the first row; the first row that ends behind one.at is the only one to look at
  const uint64_t row = one.at < behind ? 0 : (one.at - behind) / r.step + 1;
  return row < (uint64_t)r.count && r.at + row * r.step < end;
}

// Sizes and numbers, which the workspace depends on; calls: in one launch
ttc_status_t check_sizes(const ttc_linear_attention_t& a, int calls) {
  if (a.sequences < 0 || a.tokens < 0 || a.heads < 1 || a.heads_qk < 1 || a.heads % a.heads_qk || !known_dtype(a.dtype) || a.max_q < 0 || !isfinite(a.scale))
    return TTC_ERR_INVALID_ARG;
  if (!a.cu_q && a.tokens != a.sequences) return TTC_ERR_INVALID_ARG;
  if (a.dk < 8 || a.dk > 256 || a.dk % 8 || a.dv < 8 || a.dv > 256 || a.dv % 8) return TTC_ERR_UNSUPPORTED;
  // a launch has less than 2^32 threads: 512 for every head of 64 tokens, and for every 64 columns of a sequence's heads 256 in each call (of an odd number of
  // 64 columns as many as for the next even one)
  const double launch = 4294967296., slices = ((a.dk > a.dv ? a.dk : a.dv) + 63) / 64;
  if (a.tokens > 0x7fffffffll || a.sequences > 0x7fffffffll || ((double)a.tokens / 64 + a.sequences + 8) * a.heads * 512 >= launch ||
      calls * ((double)a.sequences + 8) * a.heads * (slices + 1) * 256 >= launch) return TTC_ERR_UNSUPPORTED;
  // 64 rows of a chunk lie within 2^31 bytes
  for (int64_t step : {a.q_token, a.k_token, a.v_token, a.out_token})
    if (a.tokens > 1 && (step < 0 || step >= (1 << 23))) return TTC_ERR_UNSUPPORTED;
  return TTC_OK;
}

ttc_status_t check_pointers(const ttc_linear_attention_t& a) {
  const uint64_t n = bytes_of(a.dtype);
  if (a.tokens && (!a.q || !a.k || !a.v || !a.log_decay || !aligned(a.q, n) || !aligned(a.k, n) || !aligned(a.v, n) || !aligned(a.log_decay, 4)))
    return TTC_ERR_INVALID_ARG;
  if (!aligned(a.cu_q, 4) || !aligned(a.state_row, 4) || !aligned(a.kv_len, 4) || !aligned(a.state_in, 16) || !aligned(a.state_out, 16) || a.state_rows < 0)
    return TTC_ERR_INVALID_ARG;
  return TTC_OK;
}

ttc_status_t check_norm(const ttc_residual_norm_t& n) {
  if (n.tokens < 0 || n.features < 1 || n.groups < 1 || n.features % n.groups || !known_dtype(n.dtype)) return TTC_ERR_INVALID_ARG;
  for (int32_t kind : {n.post, n.pre})
    if (kind != TTC_NORM_NONE && kind != TTC_NORM_RMS && kind != TTC_NORM_LAYER) return TTC_ERR_INVALID_ARG;
  if (n.gate && n.act != TTC_GATE_IDENTITY && n.act != TTC_GATE_SIGMOID && n.act != TTC_GATE_SILU) return TTC_ERR_INVALID_ARG;
  if (!(n.post_eps >= 0.f) || !(n.pre_eps >= 0.f) || !isfinite(n.post_eps) || !isfinite(n.pre_eps) || !isfinite(n.scale)) return TTC_ERR_INVALID_ARG;
  if (n.features > 16384 || n.tokens > 0x7fffffffll || (n.groups > 1 && n.features / n.groups % 8)) return TTC_ERR_UNSUPPORTED;
  const uint64_t b = bytes_of(n.dtype);
  if (n.tokens && (!n.y || !aligned(n.y, b) || !aligned(n.gate, b) || !aligned(n.residual, b))) return TTC_ERR_INVALID_ARG;
  for (const float* v : {n.post_gain, n.post_offset, n.residual_gain, n.pre_gain, n.pre_offset})
    if (!aligned(v, 4)) return TTC_ERR_INVALID_ARG;
  return TTC_OK;
}

bool rows_apart(int64_t stride, const ttc_residual_norm_t& n) { return n.tokens < 2 || stride >= n.features || -stride >= n.features; }

ttc_status_t check_norm_backward(const ttc_residual_norm_backward_t* b) {
  if (!b) return TTC_ERR_INVALID_ARG;
  const ttc_residual_norm_t& n = b->forward;
  if (const ttc_status_t s = check_norm(n); s != TTC_OK) return s;
  const uint64_t e = bytes_of(n.dtype);
  if (!aligned(b->gr, e) || !aligned(b->gh, e) || !aligned(b->gy, e) || !aligned(b->ggate, e) || !aligned(b->gresidual, e)) return TTC_ERR_INVALID_ARG;
  if (n.tokens && (b->gh != nullptr) != (n.pre != TTC_NORM_NONE)) return TTC_ERR_INVALID_ARG;
  if ((b->ggate && !n.gate) || (b->gresidual && !n.residual)) return TTC_ERR_INVALID_ARG;
  const float* given[5] = {n.post ? n.post_gain : nullptr, n.post ? n.post_offset : nullptr, n.residual_gain, n.pre ? n.pre_gain : nullptr,
                           n.pre ? n.pre_offset : nullptr};
  const float* wanted[5] = {b->gpost_gain, b->gpost_offset, b->gresidual_gain, b->gpre_gain, b->gpre_offset};
  for (int i = 0; i < 5; ++i)
    if (wanted[i] && (!aligned(wanted[i], 4) || (n.tokens && !given[i]))) return TTC_ERR_INVALID_ARG;
  return TTC_OK;
}

ttc_status_t check_backward(const ttc_linear_attention_backward_t* b) {
  if (!b) return TTC_ERR_INVALID_ARG;
  const ttc_linear_attention_t& f = b->forward;
  if (const ttc_status_t s = check_sizes(f, 2); s != TTC_OK) return s;
  if (f.tokens > 1 && (int64_t)f.heads * (f.dk > f.dv ? f.dk : f.dv) >= (1 << 23)) return TTC_ERR_UNSUPPORTED;  // the results' rows
  return check_pointers(f);
}

// A result in the place of another, or of rows or vectors that are read, unless the rows are the same: a thread writes its part of a row after it read it
bool norm_backward_overlaps(const ttc_residual_norm_backward_t& b) {
  const ttc_residual_norm_t& n = b.forward;
  const uint64_t e = bytes_of(n.dtype), vector = (uint64_t)n.features * 4, rows = (uint64_t)n.tokens * n.features * e;
  const Rows result[8] = {whole(b.gy, rows), whole(b.ggate, rows), whole(b.gresidual, rows), whole(b.gpost_gain, vector), whole(b.gpost_offset, vector),
                          whole(b.gresidual_gain, vector), whole(b.gpre_gain, vector), whole(b.gpre_offset, vector)};
  const void* const given[5] = {n.y, n.gate, n.residual, b.gr, b.gh};
  const int64_t stride[5] = {n.y_token, n.gate_token, n.residual_token, b.gr_token, b.gh_token};
  for (int i = 0; i < 8; ++i) {
    for (int k = 0; k < i; ++k)
      if (meet(result[i], result[k])) return true;
    if (i >= 3) continue;  // (vectors are written by a launch that reads the workspace alone)
    for (int k = 0; k < 5; ++k) {
      const bool same = result[i].at == (uint64_t)given[k] && (n.tokens < 2 || stride[k] == n.features);
      if (!same && meet(result[i], rows_of(given[k], n.tokens, stride[k], 1, 0, n.features, e))) return true;
    }
    for (const float* v : {n.post_gain, n.post_offset, n.residual_gain, n.pre_gain, n.pre_offset})
      if (meet(result[i], whole(v, vector))) return true;
  }
  return false;
}

// A result in the place of something that a later launch of the call reads, or of another result
bool backward_overlaps(const ttc_linear_attention_backward_t& b) {
  const ttc_linear_attention_t& f = b.forward;
  const uint64_t n = bytes_of(f.dtype), state = (uint64_t)f.heads * f.dk * f.dv * 4;
  const Rows result[5] = {whole(b.gq, (uint64_t)f.tokens * f.heads_qk * f.dk * n), whole(b.gk, (uint64_t)f.tokens * f.heads_qk * f.dk * n),
                          whole(b.gv, (uint64_t)f.tokens * f.heads * f.dv * n), whole(b.glog_decay, (uint64_t)(f.g_token ? f.tokens : 1) * f.heads * 4),
                          whole(b.gstate, f.sequences * state)};
  const Rows read[10] = {rows_of(f.q, f.tokens, f.q_token, f.heads_qk, f.q_head, f.dk, n), rows_of(f.k, f.tokens, f.k_token, f.heads_qk, f.k_head, f.dk, n),
                         rows_of(f.v, f.tokens, f.v_token, f.heads, f.v_head, f.dv, n), rows_of(b.gout, f.tokens, b.gout_token, f.heads, b.gout_head, f.dv, n),
                         rows_of(f.log_decay, f.tokens, f.g_token, f.heads, f.g_head, 1, 4), whole(f.state_in, f.state_rows * state),
                         whole(b.gstate_out, f.sequences * state), whole(f.cu_q, (f.sequences + 1) * 4), whole(f.state_row, f.sequences * 4),
                         whole(f.kv_len, f.sequences * 4)};
  for (int i = 0; i < 5; ++i) {
    for (const Rows& r : read)
      if (meet(result[i], r)) return true;
    for (int k = 0; k < i; ++k)
      if (meet(result[i], result[k])) return true;
  }
  return false;
}

}  // namespace

extern "C" {

size_t ttc_linear_attention_workspace_bytes(const ttc_linear_attention_t* a) {
  return a && check_sizes(*a, 1) == TTC_OK ? ttc::linear_attention_workspace(*a, ttc::compute_units()) : 0;
}

ttc_status_t ttc_linear_attention(const ttc_linear_attention_t* a, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!a) return TTC_ERR_INVALID_ARG;
  if (const ttc_status_t s = check_sizes(*a, 1); s != TTC_OK) return s;
  if (const ttc_status_t s = check_pointers(*a); s != TTC_OK) return s;
  if (a->tokens && (!a->out || !aligned(a->out, bytes_of(a->dtype)) || a->out == a->q || a->out == a->k || a->out == a->v)) return TTC_ERR_INVALID_ARG;
  if (!a->sequences || (!a->state_out && (!a->tokens || !a->max_q))) return TTC_OK;
  const uint64_t need = ttc::linear_attention_workspace(*a, ttc::compute_units());
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return TTC_ERR_WORKSPACE;
  return ttc::launch_linear_attention(*a, ttc::compute_units(), workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

size_t ttc_linear_attention_backward_workspace_bytes(const ttc_linear_attention_backward_t* b) {
  return check_backward(b) == TTC_OK ? ttc::linear_attention_backward_workspace(*b, ttc::compute_units()) : 0;
}

ttc_status_t ttc_linear_attention_backward(const ttc_linear_attention_backward_t* b, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const ttc_status_t s = check_backward(b); s != TTC_OK) return s;
  const ttc_linear_attention_t& f = b->forward;
  const uint64_t n = bytes_of(f.dtype);
  if (f.tokens && (!b->gout || !b->gq || !b->gk || !b->gv || !aligned(b->gout, n) || !aligned(b->gq, n) || !aligned(b->gk, n) || !aligned(b->gv, n)))
    return TTC_ERR_INVALID_ARG;
  if (((f.tokens || !f.g_token) && !b->glog_decay) || !aligned(b->glog_decay, 4) || !aligned(b->gstate_out, 16) || !aligned(b->gstate, 16)) return TTC_ERR_INVALID_ARG;
  if (f.tokens > 1 && (b->gout_token < 0 || b->gout_token >= (1 << 23))) return TTC_ERR_UNSUPPORTED;
  const uint64_t need = ttc::linear_attention_backward_workspace(*b, ttc::compute_units());
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return TTC_ERR_WORKSPACE;
  if (backward_overlaps(*b)) return TTC_ERR_INVALID_ARG;
  return ttc::launch_linear_attention_backward(*b, ttc::compute_units(), workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

ttc_status_t ttc_residual_norm(const ttc_residual_norm_t* n, void* hip_stream) {
  if (!n) return TTC_ERR_INVALID_ARG;
  if (const ttc_status_t s = check_norm(*n); s != TTC_OK) return s;
  if (!n->tokens) return TTC_OK;
  const uint64_t b = bytes_of(n->dtype);
  if (!aligned(n->r, b) || !aligned(n->h, b) || (n->h != nullptr) != (n->pre != TTC_NORM_NONE) || (!n->r && !n->h) || n->r == n->h) return TTC_ERR_INVALID_ARG;
  if ((n->r && !rows_apart(n->r_token, *n)) || (n->h && !rows_apart(n->h_token, *n))) return TTC_ERR_INVALID_ARG;
  const void* in[3] = {n->y, n->gate, n->residual};
  const int64_t stride[3] = {n->y_token, n->gate_token, n->residual_token};
  for (int i = 0; i < 3; ++i)
    if (in[i] && ((in[i] == n->r && stride[i] != n->r_token) || (in[i] == n->h && stride[i] != n->h_token))) return TTC_ERR_INVALID_ARG;
  return ttc::launch_residual_norm(*n, ttc::compute_units(), static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

size_t ttc_residual_norm_backward_workspace_bytes(const ttc_residual_norm_backward_t* b) {
  return check_norm_backward(b) == TTC_OK ? ttc::norm_backward_workspace(*b, ttc::compute_units()) : 0;
}

ttc_status_t ttc_residual_norm_backward(const ttc_residual_norm_backward_t* b, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (const ttc_status_t s = check_norm_backward(b); s != TTC_OK) return s;
  const uint64_t need = ttc::norm_backward_workspace(*b, ttc::compute_units());
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return TTC_ERR_WORKSPACE;
  if (norm_backward_overlaps(*b)) return TTC_ERR_INVALID_ARG;
  return ttc::launch_residual_norm_backward(*b, ttc::compute_units(), workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? TTC_OK : TTC_ERR_DEVICE;
}

}  // extern "C"
