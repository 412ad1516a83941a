/*
 * ttc_memory.h -- C ABI of the memory layers that a decoder has beside Test-Time Control blocks (the paper's hybrid, Sec. 4): linear
 * attention whose state fades by a decay of each head, with its gradients, and the norms, the gate and the residual scale that stand
 * around such a layer, an attention or a block.
 *
 * Conventions are those of ttc_attention.h: DEVICE pointers on the current device, caller-owned outputs and workspaces, no allocation, no
 * synchronisation, asynchronous launches on `hip_stream`; argument errors are reported by the return code and nothing is launched.  dtype is a
 * ttc_dtype_t (float32 or bfloat16).  Strides are in elements and need no alignment beyond the element's own (rows of 16-byte
 * alignment are read faster); the entries of one head, or of one token's features, lie side by side.
 */
#ifndef TTC_MEMORY_H
#define TTC_MEMORY_H

#include "ttc_lqr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear attention ---------------------------------------------------------------------------------------------------
 * Every head of every sequence has a state S of (dk, dv) float32 numbers.  Token t lets it fade, adds its key and value, and asks:
 *     S_t = exp(g_t) S_{t-1} + k_t v_t^T,     out_t = scale * S_t^T q_t.
 * g is the log decay, in float32, at most 0 (a positive one lets the state grow; numbers may then pass the largest float32; one below -200 counts
 * as -200, which leaves nothing of a finite state: -inf begins anew).  Head h has query and key head h / (heads / heads_qk).
 * Sequences are packed as in ttc_attention: sequence s has the rows cu_q[s] .. cu_q[s+1]-1, rows behind the last are left as they are.
 * dk and dv are multiples of 8 from 8 to 256; rows of tokens are at most 2^23 - 1 entries apart (in gradients
 * heads * max(dk, dv) too).  A launch counts 2^32 threads: (tokens / 64 + sequences + 8) * heads below 2^23 with
 * (sequences + 8) * heads below 2^20 are always taken.
 * States, sums and decays are float32 or wider.  bfloat16 rows, in gradients and where max_q is more than 6: what queries meet of the state, and the
 * products of queries and keys of one chunk of 64 tokens, are sums of two bfloat16 numbers for their products (2^-16 of each is lost); nothing
 * else but the results, gradients of decays included, is rounded to less than float32's 24 bits.
 * A token's NaN or infinity reaches its own and later tokens' results, and no earlier ones (an infinity may become NaN there). */
typedef struct {
  int64_t sequences, tokens;   /* tokens: rows of q, k, v, out; below 2^31                                 */
  int32_t heads, heads_qk;     /* heads a multiple of heads_qk                                             */
  int32_t dk, dv;
  int32_t dtype;               /* of q, k, v, out                                                          */
  int32_t max_q;               /* no sequence has more tokens (those behind it are left out)               */
  float scale;                 /* finite                                                                   */
  const void *q, *k;           /* (tokens, heads_qk, dk) by the strides below                              */
  const void *v;               /* (tokens, heads, dv)                                                      */
  void *out;                   /* (tokens, heads, dv); must not overlap the others                         */
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
  const float *log_decay;      /* token t, head h: log_decay[t*g_token + h*g_head]; g_token = 0: a head's own for all tokens */
  int64_t g_token, g_head;
  const int32_t *cu_q;         /* (sequences + 1), or NULL: one token each, tokens = sequences             */
  /* States: (state_rows, heads, dk, dv) contiguous float32, 16-byte aligned.  Sequence s has row state_row[s] (NULL: row s).  It begins with
   * what state_in has there, or with zeros where state_in is NULL, where kv_len[s] (its tokens, those of this call included) is no more
   * than its tokens in this call, or where the row lies outside; it leaves its state in the row of state_out (NULL: it is dropped; a row
   * outside: likewise).  state_out may be state_in.  No row twice in one call.  A sequence without tokens here leaves what it began with. */
  const float *state_in;
  float *state_out;
  int64_t state_rows;
  const int32_t *state_row;    /* (sequences) or NULL                                                      */
  const int32_t *kv_len;       /* (sequences) or NULL: all go on from their states                         */
} ttc_linear_attention_t;

/* workspace: DEVICE, 16-byte aligned, at least ttc_linear_attention_workspace_bytes(attention) bytes (0: none needed, may be NULL), which
 * depends on sizes and dtype and on the device's compute units alone.  It need not be cleared and may be used again by the next call on the
 * same stream.  Equal calls give equal bits. */
size_t ttc_linear_attention_workspace_bytes(const ttc_linear_attention_t *attention);
ttc_status_t ttc_linear_attention(const ttc_linear_attention_t *attention, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Gradients of a loss from dl/dout and dl/dS of the sequences' last states.  `forward` describes the forward call; its out, state_out are
 * not used.  gq, gk sum over the heads that share them; a glog_decay for g_token = 0 sums over all tokens (else it is one per token and
 * head).  gstate: with respect to the states that the sequences began with, 0 where a sequence began with zeros by rule.
 * A decay below -104, which leaves nothing of a state in float32, has the gradient 0; the others are sums over a sequence's tokens, 2^-24 of their terms off, and a
 * token's NaN or infinity may reach those of all tokens of its sequence and head (of gq, gk, gv those that depend on it; a decay's NaN any of them).  No result may
 * overlap another or anything that is read (TTC_ERR_INVALID_ARG): rows are read again after results have been written. */
typedef struct {
  ttc_linear_attention_t forward;
  const void *gout;            /* (tokens, heads, dv) of dtype by gout_token, gout_head                     */
  int64_t gout_token, gout_head;
  const float *gstate_out;     /* (sequences, heads, dk, dv) contiguous, 16-byte aligned, or NULL: zeros     */
  void *gq, *gk, *gv;          /* contiguous, of dtype: (tokens, heads_qk, dk) twice, (tokens, heads, dv)    */
  float *glog_decay;           /* contiguous: (tokens, heads), or (heads) where forward.g_token is 0         */
  float *gstate;               /* (sequences, heads, dk, dv) contiguous, 16-byte aligned, or NULL            */
} ttc_linear_attention_backward_t;
size_t ttc_linear_attention_backward_workspace_bytes(const ttc_linear_attention_backward_t *backward);
ttc_status_t ttc_linear_attention_backward(const ttc_linear_attention_backward_t *backward, void *workspace, size_t workspace_bytes,
                                           void *hip_stream);

/* ---- norms around a block --------------------------------------------------------------------------------------------------
 * What a block (attention, memory layer, TTC block) gives is normed, gated, scaled, added to the features that went past it, and normed again
 * for the next block:
 *     z = N_post(y),   u = act(gate) * z,   r = residual + scale * residual_gain * u,   h = N_pre(r),
 * every part of it optional.  N(x) = gain * (x - m) / sqrt(mean (x - m)^2 + eps) + offset, m the mean (layer norm) or 0 (rms).  N_post norms
 * each of `groups` equal parts of the features for itself (a memory layer's heads).  h comes from r before r is rounded to its type.
 * All arithmetic is float32. */
typedef enum { TTC_NORM_NONE = 0, TTC_NORM_RMS = 1, TTC_NORM_LAYER = 2 } ttc_norm_t;
typedef enum { TTC_GATE_IDENTITY = 0, TTC_GATE_SIGMOID = 1, TTC_GATE_SILU = 2 } ttc_gate_t;  /* act(x) = x, 1/(1+exp(-x)), x/(1+exp(-x)) */

typedef struct {
  int64_t tokens;
  int32_t features;            /* 1 .. 16384                                                               */
  int32_t groups;              /* 1, or parts of a multiple of 8 features                                  */
  int32_t dtype;               /* of y, gate, residual, r, h                                               */
  int32_t post, pre;           /* ttc_norm_t                                                               */
  int32_t act;                 /* ttc_gate_t; counts where there is a gate                                 */
  float post_eps, pre_eps;     /* >= 0, finite                                                             */
  float scale;                 /* finite                                                                   */
  const void *y, *gate, *residual;  /* (tokens, features) by the strides below; gate, residual may be NULL (without a residual r = scale ..) */
  void *r, *h;                 /* likewise; h NULL exactly where pre is TTC_NORM_NONE, r may be NULL where it is not.  r or h may be y, gate or
                                  residual with its stride; nothing may overlap otherwise. */
  int64_t y_token, gate_token, residual_token, r_token, h_token;
  const float *post_gain, *post_offset, *residual_gain, *pre_gain, *pre_offset;  /* (features) each, or NULL: 1, 0, 1, 1, 0 */
} ttc_residual_norm_t;
ttc_status_t ttc_residual_norm(const ttc_residual_norm_t *norm, void *hip_stream);

/* Gradients of a loss from dl/dr and dl/dh.  `forward` describes the forward call; its r and h are not used.  Any result may be NULL; a vector's
 * is summed over the tokens, in an order that depends on the sizes alone.  workspace as above.  gy, ggate, gresidual may be y, gate, residual, gr
 * or gh where these are contiguous; they may not overlap them otherwise, nor another result, nor a vector (TTC_ERR_INVALID_ARG). */
typedef struct {
  ttc_residual_norm_t forward;
  const void *gr, *gh;         /* (tokens, features) of dtype by the strides below; gr may be NULL (zeros), gh is NULL exactly where pre is none */
  int64_t gr_token, gh_token;
  void *gy, *ggate, *gresidual;    /* (tokens, features) contiguous, of dtype; a gate's is each token's, also where all tokens have the same */
  float *gpost_gain, *gpost_offset, *gresidual_gain, *gpre_gain, *gpre_offset;  /* (features); only where the forward call has the vector */
} ttc_residual_norm_backward_t;
size_t ttc_residual_norm_backward_workspace_bytes(const ttc_residual_norm_backward_t *backward);
ttc_status_t ttc_residual_norm_backward(const ttc_residual_norm_backward_t *backward, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TTC_MEMORY_H */
