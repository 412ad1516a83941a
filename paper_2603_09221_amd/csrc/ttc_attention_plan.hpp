// How the attention over the cache is shared between workgroups: row tiles, spans of the context, and the workspace where the spans'
// results meet.  Host code; the kernels read the same numbers.
#pragma once
#include <stdint.h>

#include "../../include/ttc_attention.h"

namespace ttc {

constexpr int ATT_ROWS = 16;   // query rows (new tokens x query heads of one cache head) of a workgroup
constexpr int ATT_STEP = 64;   // tokens that a wavefront takes at a time
constexpr int ATT_WAVES = 4;   // wavefronts of a workgroup, side by side along the context

struct AttentionArgs {
  ttc_attention_t a;
  int32_t group;       // query heads of one cache head
  int32_t row_tiles;   // of ATT_ROWS rows, for the longest sequence
  int32_t span;        // tokens of the context that one workgroup takes
  int32_t spans;       // for the longest context; with 1 the workgroup writes out itself
  int64_t items;       // sequences * heads * row_tiles
  int32_t join_rows;   // rows of a tile that can be real
  float *part_out;     // (items, spans, ATT_ROWS, d) sums of exp2(s - m) v
  float *part_stat;    // (items, spans, 2, ATT_ROWS): m, sum of exp2(s - m)
};

// Tokens of the context that the rows of one tile can see between them, at most
inline int64_t visible_at_most(const ttc_attention_t& a, int group) {
  if (!a.causal || !a.window) return a.max_kv;
  const int64_t tokens = (ATT_ROWS - 1) / group + 2;  // new tokens whose rows one tile holds
  const int64_t n = (int64_t)a.window + tokens + ATT_STEP;
  return n < a.max_kv ? n : a.max_kv;
}

inline void plan_attention(AttentionArgs& p, int cus) {
  const ttc_attention_t& a = p.a;
  p.group = a.heads_q / a.cache.heads;
  const int64_t rows = (int64_t)a.max_q * p.group;
  p.row_tiles = (int32_t)((rows + ATT_ROWS - 1) / ATT_ROWS);
  p.items = a.sequences * a.cache.heads * p.row_tiles;
  const int64_t most = visible_at_most(a, p.group), unit = ATT_STEP * ATT_WAVES;
  const int64_t units = (most + unit - 1) / unit;
  // about sixteen workgroups to a compute unit, as long as each has a step for every wavefront
  int64_t spans = p.items > 0 ? (16 * cus + p.items - 1) / p.items : 1;
  spans = spans < 1 ? 1 : spans > units ? units : spans;
  const int64_t per = spans ? (units + spans - 1) / spans : 1;
  p.span = (int32_t)((per < 1 ? 1 : per) * unit);
  p.spans = (int32_t)((most + p.span - 1) / p.span);
  if (p.spans < 1) p.spans = 1;
  p.join_rows = (int32_t)(rows < ATT_ROWS ? rows : ATT_ROWS);
  p.part_out = p.part_stat = nullptr;
}

inline uint64_t attention_workspace(const AttentionArgs& p) {
  return p.spans <= 1 ? 0 : (uint64_t)p.items * p.spans * ATT_ROWS * (p.a.cache.d + 2) * sizeof(float);
}

}  // namespace ttc
