// How the attention over the cache is shared between workgroups, and the workspace where their results meet.  Host code; the kernels read
// the same numbers.
#pragma once
#include <stdint.h>

#include "../../include/ttc_attention.h"

namespace ttc {

constexpr int ATT_ROWS = 16;   // query rows (new tokens x query heads of one cache head) of a tile
constexpr int ATT_STEP = 64;   // tokens that a wavefront takes at a time
constexpr int ATT_WAVES = 4;   // wavefronts of a workgroup, side by side along the context
constexpr int ATT_UNIT = ATT_STEP * ATT_WAVES;

constexpr int PROMPT_WAVES = 4;  // wavefronts of a workgroup of the kernel for many rows, 32 rows each
// It keeps operands, sums and a step's weights of 32 rows in registers.  Queries of three parts, or heads of 256, do not fit: with float32 and
// d = 128 it took 463 us where attention_kernel takes 369 (64 cache heads, 4096 rows each over 1024 tokens), with bfloat16 and d = 256 it was
// at most 1.28 times faster, so those shapes do without.
constexpr bool prompt_kernel(bool bf16, int d) { return d == 64 || (bf16 && d == 128); }

// Workgroups that a compute unit holds at once, by the registers that a wavefront needs; d = 64 / 128 / 256.  Measured with one / two / three (us;
// with three, d = 128 spills, as d = 256 does with two): bfloat16, 64 sequences of 257 to 16384 tokens at d = 64 140 / 95 / 77, four of 65536
// at d = 128 73 / 55 / 68, four of 32768 at d = 256 61 / 98 / 97.
constexpr int att_resident(int d) { return d == 64 ? 3 : d == 128 ? 2 : 1; }

struct AttentionArgs {
  ttc_attention_t a;
  int32_t group;       // query heads of one cache head
  int32_t row_tiles;   // of ATT_ROWS rows, for the longest sequence
  int32_t entries;     // sequences * row_tiles
  int64_t items;       // entries * heads: what one workgroup would do by itself
  int32_t prompt;      // whether the kernel for many rows is taken; row_tiles are its own then
  int32_t shared;      // whether the workgroups share the items' units evenly; else each does an item
  int64_t workgroups;
  float *part_out;     // (2 * workgroups, ATT_ROWS, d) sums of exp2(s - m) v
  float *part_stat;    // (2 * workgroups, ATT_ROWS, 2): m, sum of exp2(s - m)
  unsigned long long *marks;  // (2 * workgroups): which slots are written
  unsigned long long mark;    // the call's own
};

// Tokens of the context that the rows of one tile can see between them, at most
inline int64_t visible_at_most(const ttc_attention_t& a, int group) {
  if (!a.causal || !a.window) return a.max_kv;
  const int64_t tokens = (ATT_ROWS - 1) / group + 2;  // new tokens whose rows one tile holds
  const int64_t n = (int64_t)a.window + tokens + ATT_STEP;
  return n < a.max_kv ? n : a.max_kv;
}

// Shared: the contexts are cut into units of 256 tokens and every workgroup that the device holds at once gets the same number of
// them, whatever the sequences' lengths; an item whose units several workgroups have is joined by the last of them.  Otherwise each item is a
// workgroup's own, which the device deals out as others end: no join and no sum over the lengths, but the longest item is the least
// time (2 us a unit).  Shared pays where that item is long next to what a compute unit gets.  Measured, shared / own, us: d = 128
// bfloat16, 32 items of 1000 tokens 15.4 / 13.1, of 4099 17.9 / 36; 512 items of 2000 30 / 29, of 8000 91 / 93, of 0 to 2000 32 / 24, of
// 0 to 8000 68 / 74; d = 64 float32, 2048 items of 4099 184 / 158.  (Lengths of all sequences but one near 0 would move the balance to sharing:
// hence 4 units for every item of a compute unit, where even lengths would allow 8.)
// False: more than the kernels' counters or one launch hold (numbers of tokens and rows are 32-bit inside a sequence, and so are tiles of a head; a
// launch has fewer than 2^24 workgroups).  max_q may be far above what the sequences have: workgroups of the kernel for many rows, and
// those that share, do not grow with it.
inline bool plan_attention(AttentionArgs& p, int cus) {
  p.group = p.a.heads_q / p.a.cache.heads;
  if (p.a.max_kv > (1 << 30) || (int64_t)p.a.max_q * p.group > (1 << 30)) return false;
  // A cache of no pages holds no tokens, and there is none to read in the place of a page that is missing.
  if (!p.a.cache.pages) p.a.max_kv = 0;
  // Without cu_q every sequence has one row, however wide the bound: tiles are counted by it, in the grid and in the kernels.
  if (!p.a.cu_q && p.a.max_q > 1) p.a.max_q = 1;
  const ttc_attention_t& a = p.a;
  const int64_t rows = (int64_t)a.max_q * p.group;
  const double most = (double)a.sequences * ((double)rows / ATT_ROWS + 1);
  if (most >= 2147483648. || most * a.cache.heads >= 1e15) return false;
  // The kernel for many rows does a tile's context from end to end in one workgroup: 1.2 us for every 64 tokens, however few of its 128
  // rows there are, up to a tile to each compute unit; attention_kernel takes tiles of 16 in time proportional to their number.  So there have to
  // be rows for three quarters of the compute units' tiles, and half a tile of them to a sequence; with float32 for all, and three quarters of one.
  // This one / attention_kernel, us.  By the first condition, d = 128, one sequence over 8192 tokens, rows for 64 tiles 193 / 90, 128
  // 197 / 161, 256 210 / 304; 256 sequences of 8192 tokens with 64 rows 205 / 203, 96 205 / 296.  By the second, 1024 items (128 sequences, 8
  // cache heads) of 600 tokens, 32 rows 67 / 47, 64 72 / 86, 80 75 / 106; d = 64, 512 sequences of 8192 tokens, 64 rows 231 / 242, 92 233 / 355;
  // float32, d = 64, 1024 items of 600 tokens, 64 rows 86 / 74, 96 92 / 106.  The host knows no lengths: where they are far apart the longest
  // is this one's time, and 512 sequences of 0 to 8192 tokens with 64 rows take 206 / 160.  One bound and one choice for all sequences of a
  // call: single tokens beside a long chunk are taken as the chunk is.
  const bool bf16 = a.dtype == TTC_BF16;
  const int64_t prompt_tiles = (rows + 32 * PROMPT_WAVES - 1) / (32 * PROMPT_WAVES);
  const int64_t all_rows = (a.tokens < a.sequences * a.max_q ? a.tokens : a.sequences * a.max_q) * p.group;
  const int64_t tiles = a.sequences * prompt_tiles, real = all_rows / (32 * PROMPT_WAVES) + a.sequences;
  p.prompt = prompt_kernel(bf16, a.cache.d) && a.cache.heads * all_rows >= (bf16 ? 96 : 128) * (int64_t)cus &&
             all_rows >= (bf16 ? 64 : 96) * a.sequences;
  const int tile = p.prompt ? 32 * PROMPT_WAVES : ATT_ROWS;
  p.row_tiles = (int32_t)((rows + tile - 1) / tile);
  p.entries = (int32_t)(a.sequences * p.row_tiles);
  p.items = (int64_t)p.entries * a.cache.heads;
  const int64_t slots = (int64_t)att_resident(a.cache.d) * cus;
  const int64_t units = (visible_at_most(a, p.group) + ATT_UNIT - 1) / ATT_UNIT;
  const int64_t own = 4 * p.items / cus;
  // (entries: every wavefront adds up their units, 16 to a lane at most.  The empty tiles of a long max_q count among them.)
  p.shared = !p.prompt && units > (own > 4 ? own : 4) && p.entries <= 1024 && (double)units * p.items < 1e9;
  p.workgroups = p.prompt ? a.cache.heads * (tiles < real ? tiles : real) : !p.shared ? p.items : units * p.items < slots ? units * p.items : slots;
  p.part_out = p.part_stat = nullptr;
  p.marks = nullptr;
  p.mark = 0;
  return p.workgroups < (1 << 24);
}

inline uint64_t attention_workspace(const AttentionArgs& p) {
  return p.shared ? 2 * (uint64_t)p.workgroups * (ATT_ROWS * (p.a.cache.d + 2) * sizeof(float) + sizeof(*p.marks)) : 0;
}

inline void place_workspace(AttentionArgs& p, void* workspace, uint64_t mark) {
  if (!p.shared) return;
  p.part_out = static_cast<float*>(workspace);
  p.part_stat = p.part_out + 2 * (uint64_t)p.workgroups * ATT_ROWS * p.a.cache.d;
  p.marks = reinterpret_cast<unsigned long long*>(p.part_stat + 2 * (uint64_t)p.workgroups * ATT_ROWS * 2);
  p.mark = mark;
}

}  // namespace ttc
