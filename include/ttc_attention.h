/*
 * ttc_attention.h -- C ABI of what stands in front of a Test-Time Control block in a decoder layer (the paper's hybrid of
 * memory layers and the block, Sec. 4): rotary positions, a paged key-value cache held in 4 bits, and attention over it.
 *
 * Conventions are those of ttc_lqr.h: DEVICE pointers, caller-owned outputs and workspaces, no allocation, no
 * synchronisation, asynchronous launches on `hip_stream`; argument errors are reported by the return code and nothing is
 * launched.  dtype is a ttc_dtype_t (float32 or bfloat16); all arithmetic is float32 or wider unless stated.  Strides are in
 * elements and need no alignment beyond the element's own (rows of 16-byte alignment are read faster); the entries of one
 * head lie side by side.
 */
#ifndef TTC_ATTENTION_H
#define TTC_ATTENTION_H

#include "ttc_lqr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rotary positions ------------------------------------------------------------------------------------------------
 * The first `rot` entries of every head are rot/2 pairs; pair i of a token at position p is turned by the angle p * f_i:
 *     a' = a cos - b sin,   b' = b cos + a sin.
 * The entries behind them are copied.  cos and sin come from a float32 table (table_rows, rot/2, 2), one row per position,
 * which ttc_rope_table fills; scaling for contexts longer than those trained on is a choice of the f_i and of the table's scale. */
typedef enum {
  TTC_ROPE_HALF = 0,        /* pair i = entries i and i + rot/2 */
  TTC_ROPE_INTERLEAVED = 1  /* pair i = entries 2i and 2i + 1   */
} ttc_rope_layout_t;

typedef struct {
  int64_t tokens;
  int32_t heads, d;            /* heads of d entries, d >= 1                                              */
  int32_t rot;                 /* even, 0 <= rot <= d                                                     */
  int32_t dtype;               /* ttc_dtype_t of x and y                                                  */
  int32_t layout;              /* ttc_rope_layout_t                                                       */
  const void *x;               /* entry e of head h of token t: x[t*x_token + h*x_head + e]               */
  void *y;                     /* likewise; may be x itself with the same strides, must not overlap it otherwise */
  int64_t x_token, x_head, y_token, y_head;
  const int64_t *positions;    /* (tokens); one outside 0 .. table_rows-1 gives NaN in the rotated entries */
  const float *table;          /* (table_rows, rot/2, 2): cos, sin; 8-byte aligned                        */
  int64_t table_rows;
} ttc_rope_t;

/* y = x with its positions. */
ttc_status_t ttc_rope(const ttc_rope_t *rope, void *hip_stream);

/* The gradient: x is dl/dy, y receives dl/dx, which is the transposed rotation (the table's scale included). */
ttc_status_t ttc_rope_backward(const ttc_rope_t *rope, void *hip_stream);

/* table[p][i] = scale * (cos, sin)(p * freqs[i]) for p < rows, i < pairs; angles and their cosines in float64, rounded once.
 * freqs: DEVICE, float64 (pairs). */
ttc_status_t ttc_rope_table(float *table, int64_t rows, int32_t pairs, const double *freqs, double scale, void *hip_stream);

/* ---- the cache ---------------------------------------------------------------------------------------------------------
 * `pages` pages of `page` tokens each (page: 16, 32, 64, 128 or 256; heads of d = 64, 128 or 256).  Token slot s is token
 * s % page of page s / page.  Keys and values are held as blocks of 32 entries of a head: an exponent byte E and 32 codes of
 * 4 bits (bit 3 the sign, magnitudes 0 .5 1 1.5 2 3 4 6); a code c stands for c * 2^(E - 127) where E <= 252, for NaN where E is
 * larger (some codes would pass the largest float32).  4.25 bits an entry.  A cache need not be cleared: bytes that no token was
 * written to may hold anything.  One head of one page is page*(d + d/16) consecutive bytes, four parts:
 *     keys' codes      [token][d/2]                       entry e: byte e/2, the low half for even e
 *     values' codes    [token/4][16][token%4][d/32]       lane l of 16 holds entries l*d/16 ..  of four tokens side by side
 *     keys' exponents  [token][d/32]
 *     values' exponents [token/4][d/32][token%4]
 * which is the order the attention's matrix operands are read in: d/8 consecutive bytes of a token's keys are one lane's share
 * of its products, four tokens' values of one lane become its columns without an exchange between lanes. */
typedef struct {
  void *data;                  /* (pages, heads, page*(d + d/16)) bytes, 16-byte aligned */
  int64_t pages;
  int32_t heads, d, page;
} ttc_kv_cache_t;

/* Bytes of one head of one page; 0 for an unsupported d or page. */
size_t ttc_kv_page_bytes(int32_t d, int32_t page);

/* New tokens' keys and values into the cache, the keys with their positions, and (optionally) the new tokens' queries with
 * theirs, in one launch.  Rounding: a block's exponent is that of its largest magnitude f * 2^k (1 <= f < 2), k - 2, one more
 * from f = 1.75 on (the largest would round up to 8), within 0 .. 252 as a byte; codes are rounded to nearest, ties to even, and stop
 * at 6 (which only numbers from 1.75 * 2^127 on do).  A block with a NaN or an
 * infinity becomes NaN.  The rotated key is not rounded in between. */
typedef struct {
  ttc_kv_cache_t cache;
  int64_t tokens;
  int32_t dtype;               /* of k, v, q, q_out                                                        */
  int32_t rot, layout;         /* as in ttc_rope_t; rot = 0: no positions (positions and table may be NULL) */
  const void *k, *v;           /* (tokens, heads, d) by the strides below                                   */
  int64_t k_token, k_head, v_token, v_head;
  const int64_t *slots;        /* (tokens) where each goes; one outside 0 .. pages*page-1 (-1: padding) is left out.
                                  No slot twice in one call. */
  const int64_t *positions;
  const float *table;
  int64_t table_rows;
  const void *q;               /* (tokens, heads_q, d) or NULL                                             */
  void *q_out;                 /* rotated queries; may be q itself with the same strides                    */
  int32_t heads_q;
  int64_t q_token, q_head, q_out_token, q_out_head;
} ttc_kv_append_t;
ttc_status_t ttc_kv_append(const ttc_kv_append_t *append, void *hip_stream);

/* What the cache holds for n slots, as numbers: k_out, v_out (n, heads, d) contiguous, of out_dtype (both types hold every
 * number of the cache exactly); a slot outside the cache gives zeros.  k_out or v_out may be NULL. */
ttc_status_t ttc_kv_read(const ttc_kv_cache_t *cache, const int64_t *slots, int64_t n, int32_t out_dtype, void *k_out,
                         void *v_out, void *hip_stream);

/* ---- attention over the cache -------------------------------------------------------------------------------------------
 * For every sequence its new tokens' queries over the tokens that the cache holds of it, the new ones included:
 *     s_j = scale * (q . k_j) over the visible j,   lse = log sum_j exp s_j,   out = sum_j exp(s_j - lse) v_j.
 * Query head h reads cache head h / (heads_q / heads).  Query i of m new ones of a sequence of n tokens is token p = n - m + i.
 * Causal: it sees tokens j <= p, with a window w > 0 only p - w < j <= p.  Otherwise all n.  A query that sees nothing gets
 * out = 0 and lse = -inf.  What a query does not see has no influence on it, NaN included.
 * Queries of float32 are worked on as exact sums of parts, sums and statistics are float32; for bfloat16 the weights
 * exp(s_j - max) are rounded to bfloat16 for their product with the values (at most 2^-8 of sum_j exp(s_j - lse) |v_j|).  Values are
 * summed before they are divided, with weights of up to 2^8: where they are beyond 2^119 / n a sum may pass the largest float32.
 * Equal calls give equal bits; the last bits of a sequence's result may differ with the other sequences of the call, which decide how
 * its context is divided. */
typedef struct {
  ttc_kv_cache_t cache;
  int64_t sequences;
  int64_t tokens;              /* rows of q and out                                                        */
  int32_t heads_q;             /* a multiple of cache.heads                                                */
  int32_t dtype;               /* of q and out                                                             */
  int32_t causal;              /* 0 or 1                                                                   */
  int32_t window;              /* 0: none; needs causal                                                    */
  float scale;                 /* finite                                                                   */
  int32_t max_q;               /* no sequence has more new tokens (those behind it are left out)           */
  int32_t max_kv;              /* no sequence has more tokens (kv_len is read as at most this)             */
  const void *q;               /* (tokens, heads_q, d) by the strides below                                */
  void *out;                   /* likewise; must not overlap q                                             */
  float *lse;                  /* (tokens, heads_q) contiguous, or NULL                                    */
  int64_t q_token, q_head, out_token, out_head;
  const int32_t *cu_q;         /* (sequences + 1): sequence s has rows cu_q[s] .. cu_q[s+1]-1; NULL: one each, tokens = sequences */
  const int32_t *kv_len;       /* (sequences)                                                              */
  const int32_t *block_table;  /* (sequences, >= ceil(max_kv / page)): page numbers by table_stride; a page outside the cache
                                  holds no visible tokens                                                  */
  int64_t table_stride;
} ttc_attention_t;

/* workspace: DEVICE, 16-byte aligned, at least ttc_attention_workspace_bytes(attention) bytes (0: none needed, may be NULL),
 * which depends on the sizes, dtype, causal and window and on the device's compute units, on nothing that lies in device memory.  One
 * launch; the workspace need not be cleared and may be used again by the next call on the same stream. */
size_t ttc_attention_workspace_bytes(const ttc_attention_t *attention);
ttc_status_t ttc_attention(const ttc_attention_t *attention, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TTC_ATTENTION_H */
