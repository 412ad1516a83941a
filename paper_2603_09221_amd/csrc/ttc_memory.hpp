// Linear attention with a decay of each head (ttc_linear_attention, ttc_linear_attention_backward).
//
// With G_t = g_1 + .. + g_t within a chunk of 64 tokens and S the state that the chunk finds,
//     out_i = in_i (x_i S) + sum_{j <= i} exp(G_i - G_j) (x_i . w_j) v_j,     in_i = exp(G_i),
//     S    <- exp(G_64) S + sum_j w_j (up_j v_j)^T,                           up_j = exp(G_64 - G_j),
// for queries x, keys w, values v: three products of matrices.  The gradients are the same sums with other rows in these places,
//     dq: x = dout, w = v, v = k, S transposed;    dk: x = v, w = dout, v = q;    dv: x = k, w = q, v = dout,
// the last two from the last token to the first (j >= i, in_i = exp(G_64 - G_i), up_j = exp(G_j)) over the state's gradient R.  So one kernel
// does all four.
#pragma once
#include "../../include/ttc_memory.h"
#include "ttc_serve.hpp"

namespace ttc {

constexpr int MEM_CHUNK = 64;      // tokens of a chunk: a lane each where decays are added up

// ---- sequences and their segments ---------------------------------------------------------------------------------------------

struct MemSequences {
  int64_t sequences, tokens;
  const int32_t* cu_q;
  int32_t max_q;
  int32_t segment;     // chunks of a segment
  int64_t entries;     // places for segments; every sequence has one at least
  int32_t each;        // of a sequence, as many as the longest has; 0: sequences have as many as they need, one behind the other
  int32_t blocks;      // of heads: what the XCDs take in turn is a segment of one block's heads (mem_deal)
};

// The segment and head of workgroup b, of `per_head` workgroups for each.  Every eighth workgroup lies on one XCD.  An XCD takes whole segments, of all heads
// or of a block of them: rows that heads share are in its cache.  Places without a segment come last.
__device__ __forceinline__ void mem_deal(const MemSequences& m, uint32_t b, int heads, uint32_t per_head, int64_t& entry, int& head, int& rest) {
  const uint32_t inner = heads / m.blocks * per_head, turn = b / 8, item = turn / inner * 8 + b % 8, in = turn % inner;
  entry = item / m.blocks;
  head = item % m.blocks * (heads / m.blocks) + in / per_head;
  rest = in % per_head;
}

// The rows of sequence s: numbers for all lanes if s is one
__device__ __forceinline__ void mem_rows(const MemSequences& m, int64_t s, int64_t& first, int& n) {
  if (!m.cu_q) {
    first = s;
    n = s < m.tokens ? min(1, m.max_q) : 0;
    return;
  }
  first = min((int64_t)max(m.cu_q[s], 0), m.tokens);
  const int64_t end = min((int64_t)m.cu_q[s + 1], m.tokens);
  n = (int)max(min(end - first, (int64_t)m.max_q), (int64_t)0);
}
__device__ __forceinline__ int mem_segments(const MemSequences& m, int n) {
  const int chunks = (int)(((int64_t)n + MEM_CHUNK - 1) / MEM_CHUNK);
  return max(1, (chunks + m.segment - 1) / m.segment);
}

// The segment at place `at`: its sequence with that one's rows, and which of its segments it is, the same for all lanes; false if there is none.  Where
// sequences have no places of their own each wavefront adds them up for itself, a run of them to a lane; if a run is one, what the lanes have read is all
// that it takes.
__device__ __forceinline__ bool mem_segment(const MemSequences& m, int64_t at, int64_t& seq, int& segment, int64_t& first, int& n) {
  if (m.each) {
    if (at >= m.entries) return false;
    seq = (uint32_t)at / (uint32_t)m.each;
    segment = (int)((uint32_t)at % (uint32_t)m.each);
    mem_rows(m, seq, first, n);
    first = __builtin_amdgcn_readfirstlane((int)first);  // (tokens are below 2^31)
    n = __builtin_amdgcn_readfirstlane(n);
    return segment < mem_segments(m, n);
  }
  const int lane = threadIdx.x & 63;
  const int64_t run = (m.sequences + 63) / 64, own_first = min(lane * run, m.sequences), own_last = min(own_first + run, m.sequences);
  uint32_t own = 0;
  int64_t row = 0;
  int rows = 0;
  for (int64_t s = own_first; s < own_last; ++s) {
    mem_rows(m, s, row, rows);
    own += mem_segments(m, rows);
  }
  uint32_t sum = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(sum, o, 64);
    sum += lane >= o ? x : 0;
  }
  if (at >= __builtin_amdgcn_readlane(sum, 63)) return false;
  const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(at < sum));
  uint32_t before = __builtin_amdgcn_readlane(sum - own, who);
  int64_t s = who * run;
  if (run > 1) {
    for (;; ++s) {
      mem_rows(m, s, row, rows);
      const uint32_t count = __builtin_amdgcn_readfirstlane(mem_segments(m, rows));
      if (at < before + count) break;
      before += count;
    }
    first = __builtin_amdgcn_readfirstlane((int)row);
    n = __builtin_amdgcn_readfirstlane(rows);
  } else {
    first = __builtin_amdgcn_readlane((int)row, who);
    n = __builtin_amdgcn_readlane(rows, who);
  }
  seq = s;
  segment = (int)(at - before);
  return true;
}

// ---- states ---------------------------------------------------------------------------------------------------------------

struct MemStates {
  const float* in;
  float* out;
  int64_t rows;
  const int32_t* row;
  const int32_t* kv_len;
};

// Row of sequence s that it goes on from; -1: it begins with zeros
__device__ __forceinline__ int64_t mem_begin(const MemStates& t, int64_t s, int n) {
  if (!t.in || (t.kv_len && t.kv_len[s] <= n)) return -1;
  const int64_t r = t.row ? t.row[s] : s;
  return r >= 0 && r < t.rows ? r : -1;
}
__device__ __forceinline__ int64_t mem_end(const MemStates& t, int64_t s) {
  if (!t.out) return -1;
  const int64_t r = t.row ? t.row[s] : s;
  return r >= 0 && r < t.rows ? r : -1;
}

__device__ __forceinline__ float mem_decay(float g) { return g < -200.f ? -200.f : g; }  // (exp(-200) is 0 in float32; NaN stays)

// ---- operands ---------------------------------------------------------------------------------------------------------------
// A lane's share of an operand of 16 x 32 numbers: eight of row (or column) lane % 16.  float32 takes eight instructions of depth 4, whose
// k-th numbers are the lanes' k-th; which numbers of the sum these are does not matter as long as both operands agree.

template <typename T> struct MemOperand;
template <> struct MemOperand<unsigned short> { typedef srv_bf16x8 type; };
struct mem_float8 { float x[8]; };
template <> struct MemOperand<float> { typedef mem_float8 type; };

__device__ __forceinline__ srv_floatx4 mem_mma(const srv_bf16x8& a, const srv_bf16x8& b, srv_floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ srv_floatx4 mem_mma(const mem_float8& a, const mem_float8& b, srv_floatx4 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[i], b.x[i], c, 0, 0, 0);
  return c;
}

// numbers side by side at p and at q, four each
__device__ __forceinline__ srv_bf16x8 mem_operand(const unsigned short* p, const unsigned short* q) {
  const srv_uintx2 a = *reinterpret_cast<const srv_uintx2*>(p), b = *reinterpret_cast<const srv_uintx2*>(q);
  return __builtin_bit_cast(srv_bf16x8, srv_uintx4{a[0], a[1], b[0], b[1]});
}
__device__ __forceinline__ mem_float8 mem_operand(const float* p, const float* q) {
  const srv_floatx4 a = *reinterpret_cast<const srv_floatx4*>(p), b = *reinterpret_cast<const srv_floatx4*>(q);
  return {{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
// Column c of the eight rows 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3, `step` numbers apart; p: column 0 of 16 of row 0 in LDS.  Of bfloat16 sixteen
// lanes read four rows of sixteen numbers, four to a lane, and get a column's four each.
__device__ __forceinline__ srv_bf16x8 mem_column(const unsigned short* p, int step, int g, int c) {
  typedef __bf16 four_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) four_t* lds_t;
  const unsigned short* q = p + (4 * g + (c >> 2)) * step + (c & 3) * 4;
  const four_t a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_t)q), b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_t)(q + 16 * step));
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ mem_float8 mem_column(const float* p, int step, int g, int c) {
  mem_float8 x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x.x[i] = p[(4 * g + i + (i < 4 ? 0 : 12)) * step + c];
  return x;
}
__device__ __forceinline__ float mem_entry(const srv_bf16x8& v, int i) { return (float)v[i]; }
__device__ __forceinline__ float mem_entry(const mem_float8& v, int i) { return v.x[i]; }

// `so_far`, 0, or NaN if one of the numbers is not finite
__device__ __forceinline__ float mem_finite(const srv_bf16x8& v, float so_far) {
  const srv_bf16x2 none = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) so_far = __builtin_amdgcn_fdot2_f32_bf16(srv_bf16x2{v[2 * i], v[2 * i + 1]}, none, so_far, false);
  return so_far;
}
__device__ __forceinline__ float mem_finite(const mem_float8& v, float so_far) {
#pragma unroll
  for (int i = 0; i < 8; ++i) so_far = fmaf(v.x[i], 0.f, so_far);
  return so_far;
}

// Eight float32 numbers as a sum of PARTS operands, the largest part first.  One and two parts are rounded to nearest, 2^-8 and 2^-16 of a number at
// most; three are cut off and hold all 24 bits.  (An infinity leaves NaN in the second, as does a number beyond the largest bfloat16.)
template <int PARTS>
__device__ __forceinline__ void mem_split(const float (&x)[8], srv_bf16x8 (&part)[PARTS]) {
  static_assert(PARTS >= 1 && PARTS <= 3);
  if constexpr (PARTS < 3) {
#pragma unroll
    for (int i = 0; i < 8; ++i) part[0][i] = static_cast<__bf16>(x[i]);
    if constexpr (PARTS == 2)
#pragma unroll
      for (int i = 0; i < 8; ++i) part[1][i] = static_cast<__bf16>(x[i] - (float)part[0][i]);
  } else {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      srv_uintx4 p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __float_as_uint(rest[2 * i]), hi = __float_as_uint(rest[2 * i + 1]);
        p[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
        rest[2 * i] -= __uint_as_float(lo & 0xffff0000u);
        rest[2 * i + 1] -= __uint_as_float(hi & 0xffff0000u);
      }
      part[k] = __builtin_bit_cast(srv_bf16x8, p);
    }
  }
}
template <int PARTS>
__device__ __forceinline__ void mem_split(const float (&x)[8], mem_float8 (&part)[PARTS]) {
  static_assert(PARTS == 1);
#pragma unroll
  for (int i = 0; i < 8; ++i) part[0].x[i] = x[i];
}

__device__ __forceinline__ void mem_store4(unsigned short* p, const float (&x)[4]) {
  typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<u16x4*>(p) = u16x4{srv_narrow<unsigned short>(x[0]), srv_narrow<unsigned short>(x[1]), srv_narrow<unsigned short>(x[2]),
                                       srv_narrow<unsigned short>(x[3])};
}
__device__ __forceinline__ void mem_store4(float* p, const float (&x)[4]) { *reinterpret_cast<srv_floatx4*>(p) = srv_floatx4{x[0], x[1], x[2], x[3]}; }

// Eight numbers of a row, in 16-byte accesses whatever the alignment: device memory takes them at that of a number
typedef unsigned short mem_u16x8 __attribute__((ext_vector_type(8), aligned(2)));
typedef float mem_floatx4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct MemEight;
template <> struct MemEight<unsigned short> { srv_u16x8 x; };
template <> struct MemEight<float> { srv_floatx4 x[2]; };
__device__ __forceinline__ void mem_fetch(const unsigned short* p, MemEight<unsigned short>& to) { to.x = *reinterpret_cast<const mem_u16x8*>(p); }
__device__ __forceinline__ void mem_fetch(const float* p, MemEight<float>& to) {
  to.x[0] = *reinterpret_cast<const mem_floatx4*>(p);
  to.x[1] = *reinterpret_cast<const mem_floatx4*>(p + 4);
}
// to LDS, the second four `apart` from the first
template <int APART>
__device__ __forceinline__ void mem_put(unsigned short* p, const MemEight<unsigned short>& x) {
  if constexpr (APART == 4) {
    *reinterpret_cast<srv_u16x8*>(p) = x.x;
  } else {
    const srv_uintx4 u = __builtin_bit_cast(srv_uintx4, x.x);
    *reinterpret_cast<srv_uintx2*>(p) = srv_uintx2{u[0], u[1]};
    *reinterpret_cast<srv_uintx2*>(p + APART) = srv_uintx2{u[2], u[3]};
  }
}
template <int APART>
__device__ __forceinline__ void mem_put(float* p, const MemEight<float>& x) {
  *reinterpret_cast<srv_floatx4*>(p) = x.x[0];
  *reinterpret_cast<srv_floatx4*>(p + APART) = x.x[1];
}
// four numbers to a row of any alignment
__device__ __forceinline__ void mem_out4(unsigned short* p, const srv_floatx4& x) {
  typedef unsigned short u16x4 __attribute__((ext_vector_type(4), aligned(2)));
  *reinterpret_cast<u16x4*>(p) = u16x4{srv_narrow<unsigned short>(x[0]), srv_narrow<unsigned short>(x[1]), srv_narrow<unsigned short>(x[2]),
                                       srv_narrow<unsigned short>(x[3])};
}
__device__ __forceinline__ void mem_out4(float* p, const srv_floatx4& x) { *reinterpret_cast<mem_floatx4*>(p) = x; }
// and from one
template <typename T> struct MemFour { typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T)))); };

// eight numbers of a row in memory, or zeros in their place
__device__ __forceinline__ srv_bf16x8 mem_global(const unsigned short* p, bool wanted) {
  MemEight<unsigned short> x;
  mem_fetch(p, x);
  return wanted ? __builtin_bit_cast(srv_bf16x8, x.x) : srv_bf16x8{};
}
__device__ __forceinline__ mem_float8 mem_global(const float* p, bool wanted) {
  MemEight<float> x;
  mem_fetch(p, x);
  if (!wanted) x = {};
  return {{x.x[0][0], x.x[0][1], x.x[0][2], x.x[0][3], x.x[1][0], x.x[1][1], x.x[1][2], x.x[1][3]}};
}

// The sum over sixteen lanes side by side, in each of them
template <int CTRL>
__device__ __forceinline__ float mem_dpp_add(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float mem_sixteen(float x) {
  x = mem_dpp_add<0xb1>(x);     // the neighbour's
  x = mem_dpp_add<0x4e>(x);     // of two
  x = mem_dpp_add<0x141>(x);    // mirrored: of four
  return mem_dpp_add<0x140>(x); // of eight
}

// ---- the kernel of chunks ---------------------------------------------------------------------------------------------------

struct MemRows {
  const void* p;
  int64_t token, head;
  int32_t group;       // heads that share a row
  int32_t d;           // entries
};

struct MemArgs {
  MemSequences m;
  MemRows x, w, v;
  void* out;
  int64_t out_token, out_head;
  int32_t out_float;            // float32 whatever the rows' type (with dots alone)
  int32_t heads, slices;
  int32_t reverse;
  float pair_scale, in_scale, up_scale;
  const float* log_decay;
  int64_t g_token, g_head;
  MemStates states;             // of the sequences
  MemStates rule;               // whose beginning says where the last state is 0 (gstate); in NULL: no rule
  int32_t ruled;
  const float* starts;          // of the segments: (entries, heads, dk, dv), or NULL: a sequence is one segment
  float* added;                 // likewise, what a segment adds to a state that it finds as zeros (MEM_STATES)
  float* faded;                 // (entries, heads): and the factor on what it finds
  int32_t s_row, s_col;         // of a state's numbers, in elements
  int32_t dk, dv;               // rows and columns of a state as it is stored
  MemRows dot;                  // MEM_OUT_DOTS: rows whose products with what the tokens read of the state are wanted; MEM_OUT_PAIRS: those of a pair's second factor
  float* dots;                  // (slices, heads, tokens): these products, or sums of pairs
};

// Two calls of the same sizes in one launch (a gradient's, of tokens in both orders: what one leaves idle is the other's); the first `split` workgroups, a
// multiple of eight, are the first one's
struct MemTwo {
  MemArgs of[2];
  uint32_t split;
};

// Decays of a chunk, a token to a lane, added up in float64, so that the differences of sums are as exact as the decays themselves; powers of two
struct MemDecays {
  float hi[MEM_CHUNK], lo[MEM_CHUNK];   // G / ln 2 as a sum of two
  float in[MEM_CHUNK], up[MEM_CHUNK];
  float since[MEM_CHUNK], left[MEM_CHUNK];  // factors from the beginning, and to the end, of a token's sixteen (the other way round from the last token on)
  float across[4];                      // what lies across a sixteen, from its beginning to its end, / ln 2
  float whole;
};

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double mem_dpp(double x) {  // the number of another lane, 0 where there is none
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive sums over a wavefront's lanes
__device__ __forceinline__ double mem_sums(double x) {
  x += mem_dpp<0x111>(x);       // within sixteen lanes
  x += mem_dpp<0x112>(x);
  x += mem_dpp<0x114>(x);
  x += mem_dpp<0x118>(x);
  x += mem_dpp<0x142, 0xa>(x);  // what lane 15 has to the next sixteen, what lane 31 has to the upper half
  x += mem_dpp<0x143, 0xc>(x);
  return x;
}

constexpr double MEM_LOG2E = 1.4426950408889634;

// Sums of a chunk's decays in powers of two; returns the whole
__device__ __forceinline__ double mem_decays(float g, int lane, bool reverse, float in_scale, float up_scale, MemDecays& to) {
  const double sum = mem_sums((double)mem_decay(g) * MEM_LOG2E), whole = __shfl(sum, 63, 64);
  const float hi = (float)sum;
  to.hi[lane] = hi;
  to.lo[lane] = (float)(sum - hi);
  const float since = __builtin_amdgcn_exp2f(hi), left = __builtin_amdgcn_exp2f((float)(whole - sum));
  to.in[lane] = in_scale * (reverse ? left : since);
  to.up[lane] = up_scale * (reverse ? since : left);
  if (lane == 63) to.whole = since;
  const double end = __shfl(sum, lane | 15, 64), ends = __shfl(sum, (lane & 48) - 1, 64), begin = lane < 16 ? 0.0 : ends;  // (all lanes take part)
  const float after = __builtin_amdgcn_exp2f((float)(sum - begin)), ahead = __builtin_amdgcn_exp2f((float)(end - sum));
  to.since[lane] = reverse ? ahead : after;
  to.left[lane] = reverse ? after : ahead;
  if ((lane & 15) == 0) to.across[lane >> 4] = (float)(end - begin);  // not what two rounded sums differ by: sums are thousands where 16 tokens forget all
  return whole;
}
// sign: -1 where the first is the earlier one
__device__ __forceinline__ float mem_between(float a_hi, float a_lo, float b_hi, float b_lo, float sign) {
  return __builtin_amdgcn_exp2f(sign * ((a_hi - b_hi) + (a_lo - b_lo)));
}

template <typename T, int DK, int WAVES>
struct MemShape {
  // Rows of bfloat16 an odd multiple of 32 bytes apart: the columns that 32 lanes read at once lie on as many banks, and so do the 16 bytes of rows that 16
  // do.  (Of 16 bytes, with the eight rows of a column's share one behind the other: LDS was busy for 53 % of a long prompt's cycles instead of 41 %, 148 us
  // instead of 137.)  Of float32 numbers what 64 lanes read of columns lies on 64 banks with 16 bytes more.  Pairs' products are read by rows alone, with 16
  // bytes more; 16 less than the others, heads of 64 then have three workgroups of four wavefronts on a unit (64 x 32 tokens of 32 heads 34 us, else 39).
  static constexpr int PAD = sizeof(T) == 2 ? 16 : 4;
  static constexpr int COLS = 16 * WAVES;
  static constexpr int XS = DK + PAD, VS = COLS + PAD, PS = MEM_CHUNK + 16 / (int)sizeof(T);  // rows in LDS
  static constexpr int PARTS = sizeof(T) == 2 ? 2 : 1;  // of the pairs' products, one behind the other
  // the pairs' products have a place of their own unless LDS is too small for it: then that of x, for one more barrier
  static constexpr bool OWN = MEM_CHUNK * (2 * XS + VS + PARTS * PS) * sizeof(T) <= 150 * 1024;
  static constexpr int XP = DK / 8 / WAVES, VP = 2;  // pieces of eight that a thread brings
  // wavefronts of a SIMD that registers are kept for: two workgroups on a compute unit, where LDS has room for them; two at least, for with all 512
  // registers of one the compiler puts sums into accumulation registers and reads some of them too early behind a branch (the build looks for that)
  static constexpr int RESIDENT = sizeof(T) == 2 && DK <= 128 ? WAVES / 2 : 2;
  static constexpr bool AHEAD = sizeof(T) == 2 || DK * 8 <= 128 * WAVES;  // registers for the next chunk's rows
};

// Where entry e, a multiple of four, of a row of x lies in LDS: 16 b + 4 g + r at 8 g + 4 b + r of every 32, so that what a lane reads to meet a state's numbers
// lies side by side
__device__ __forceinline__ uint32_t mem_place(uint32_t e) { return (e & ~31u) + (e & 12) * 2 + (e & 16) / 4; }

// 64 rows on their way to LDS: zeros behind the last row and behind the last entry.  Those places are read from the last row and entry that
// are there, so that no load waits for a branch.
template <typename T, int D, int STEP, int PIECES, int THREADS, bool PLACED = false>
struct MemStage {
  static constexpr int ROW = D / 8, TURN = THREADS / ROW;  // pieces of a row, rows of one turn of the workgroup
  static_assert(PIECES * TURN == MEM_CHUNK);
  MemEight<T> piece[PIECES];
  // 64 rows are less than 2^31 bytes.  Places are found anew every time: kept over the loop, with their upper halves, they would take registers that spill.
  __device__ __forceinline__ void fetch(const T* at, int64_t token, int rows, int entries) {
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const uint32_t row = thread / ROW, e = thread % ROW * 8, mine = e < (uint32_t)entries ? e : 0;
    if (rows == MEM_CHUNK) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) mem_fetch(at + i * TURN * token + (row * (uint32_t)token + mine), piece[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) mem_fetch(at + (min(row + i * TURN, (uint32_t)rows - 1) * (uint32_t)token + mine), piece[i]);
    }
  }
  __device__ __forceinline__ void put(T* lds, int rows, int entries, bool whole) const {
    constexpr int APART = PLACED ? 8 : 4;
    T* p = lds + threadIdx.x / ROW * STEP + (PLACED ? mem_place(threadIdx.x % ROW * 8) : threadIdx.x % ROW * 8);
    if (whole) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) mem_put<APART>(p + i * TURN * STEP, piece[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const bool there = (int)(threadIdx.x % ROW) * 8 < entries && (int)(threadIdx.x / ROW) + i * TURN < rows;
        mem_put<APART>(p + i * TURN * STEP, there ? piece[i] : MemEight<T>{});
      }
    }
  }
};

// A wavefront's numbers of a state in memory: rows 16 k + 4 g + r of column c, `row` numbers apart
template <int KT>
struct MemPlace {
  uint32_t at;          // of the lane's first number
  int rows;             // of the state from the lane's first on; 0: it has no such column
  int row;
  __device__ __forceinline__ void load(const float* p, bool whole, srv_floatx4 (&s)[KT]) const {
    p += at;
    if (whole && row == 1) {
#pragma unroll
      for (int k = 0; k < KT; ++k) s[k] = *reinterpret_cast<const srv_floatx4*>(p + 16 * k);
    } else if (whole) {
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[k][r] = p[(16 * k + r) * row];
    } else {
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[k][r] = 16 * k + r < rows ? p[(16 * k + r) * row] : 0.f;
    }
  }
  __device__ __forceinline__ void store(float* p, bool whole, const srv_floatx4 (&s)[KT], bool none) const {
    p += at;
#pragma unroll
    for (int k = 0; k < KT; ++k)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (whole || 16 * k + r < rows) p[(16 * k + r) * row] = none ? 0.f : s[k][r];
  }
};

// What a segment adds to its state; results; results and their products with other rows; results and sums of the pairs' products with others'
enum MemWhat { MEM_STATES, MEM_OUT, MEM_OUT_DOTS, MEM_OUT_PAIRS };

// A workgroup takes one segment of one head of one sequence, and of the values' columns a slice of 16 * WAVES; a wavefront owns 16 of them and their
// state, DK numbers each, which stays in its registers from chunk to chunk: what a lane holds of it as a result is what it has to hold of it as an operand
// if the sum's order follows.  The next chunk's rows and decays are on their way while one is worked on.
// bfloat16 rows: pairs' products and the state that queries meet have two bfloat16 parts for their products, 2^-16 of each off, as the header's documentation
// states: results are then as near as their own rounding lets them (16384 tokens 0.00166 in the norm, with one part each 0.00235; two take 228 us, one 209).
// Where gradients of decays, sums of float32 numbers, depend on what a token reads, the state has three parts, all of float32's bits, and so has
// always what is added to it (two left a state of 16384 tokens 1.6e-6 off in the norm; three leave 1.3e-7).
// MEM_OUT_PAIRS: where the rows of results are keys and values (dv), a pair's product times that of the value and the result's gradient is its share of the
// decays' gradients between the two tokens: added up by rows and by columns here, where all but one operand is in LDS (a kernel of its own took 38 us of
// 250 for four times 2048 tokens of 16 heads of 128, this takes 17).
// 16384 tokens of 32 heads of 128 x 128 over 8 of queries and keys, bfloat16: 164 us, in which the matrix instructions are busy for 29 % of the cycles, the vector
// instructions for 46 %, LDS for 40 %: a workgroup's phases between its barriers need them by turns, and only two workgroups share a unit.
// Twelve sequences of up to 1500 tokens, 16 heads of 64 x 64, float32: 75 us, matrix instructions 35 %.
template <typename T, int DK, int WAVES, int WHAT>
__global__ void __launch_bounds__(64 * WAVES, (MemShape<T, DK, WAVES>::RESIDENT)) memory_chunk_kernel(const MemTwo two) {
  const bool second = blockIdx.x >= two.split;
  const MemArgs& a = two.of[second];
  typedef MemShape<T, DK, WAVES> S;
  typedef typename MemOperand<T>::type op_t;
  constexpr bool BF16 = sizeof(T) == 2, STATES = WHAT == MEM_STATES, DOTS = WHAT == MEM_OUT_DOTS;
  constexpr bool PAIRS = WHAT == MEM_OUT_PAIRS;
  constexpr int IN = !BF16 ? 1 : DOTS ? 3 : 2, UP = BF16 ? 3 : 1, KT = DK / 16;
  constexpr int HALVES = WAVES / 4;  // wavefronts that share sixteen rows of pairs
  __shared__ alignas(16) T xl[STATES ? 8 : MEM_CHUNK * (S::OWN || S::XS > S::PS ? S::XS : S::PS)], wl[MEM_CHUNK * S::XS], vl[MEM_CHUNK * S::VS];
  __shared__ alignas(16) T own[STATES || !S::OWN ? 8 : S::PARTS * MEM_CHUNK * S::PS];
  __shared__ alignas(16) MemDecays decays[2];
  __shared__ alignas(16) float meet[WAVES == 4 ? 5 : 8][MEM_CHUNK];
  T* const pl = S::OWN ? own : xl;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int c = lane & 15, g = lane >> 4;
  int64_t entry;
  int head, slice;
  mem_deal(a.m, second ? blockIdx.x - two.split : blockIdx.x, a.heads, a.slices, entry, head, slice);
  int64_t seq, first;
  int segment, n;
  if (entry >= a.m.entries || !mem_segment(a.m, entry, seq, segment, first, n)) return;
  const int chunks = (int)(((int64_t)n + MEM_CHUNK - 1) / MEM_CHUNK), segments = max(1, (chunks + a.m.segment - 1) / a.m.segment);
  const int c0 = segment * a.m.segment, c1 = min(c0 + a.m.segment, chunks);
  const bool reverse = a.reverse;
  const int order = reverse ? -1 : 1;  // (a factor, where a choice would be a branch)
  const float sign = (float)order;
  if (STATES && segment == (reverse ? 0 : segments - 1)) return;  // nobody finds what this one leaves
  const int col0 = slice * S::COLS + wave * 16, cols = a.v.d;

  MemStage<T, DK, S::XS, S::XP, 64 * WAVES, true> x_rows;
  MemStage<T, DK, S::XS, S::XP, 64 * WAVES> w_rows;
  MemStage<T, S::COLS, S::VS, S::VP, 64 * WAVES> v_rows;
  float g_next = 0.f;
  const T* const x_at = static_cast<const T*>(a.x.p) + (STATES ? 0 : head / a.x.group * a.x.head);
  const T* const w_at = static_cast<const T*>(a.w.p) + head / a.w.group * a.w.head;
  const T* const v_at = static_cast<const T*>(a.v.p) + head / a.v.group * a.v.head + slice * S::COLS;
  const auto fetch = [&](int chunk, int rows) {
    const int64_t t0 = first + (int64_t)chunk * MEM_CHUNK;
    if (!STATES) x_rows.fetch(x_at + t0 * a.x.token, a.x.token, rows, a.x.d);
    w_rows.fetch(w_at + t0 * a.w.token, a.w.token, rows, a.w.d);
    v_rows.fetch(v_at + t0 * a.v.token, a.v.token, rows, cols - slice * S::COLS);
  };
  const auto fetch_decays = [&](int chunk, int rows) {
    g_next = a.log_decay[(first + (int64_t)chunk * MEM_CHUNK + min(lane, rows - 1)) * a.g_token + head * a.g_head];
  };
  const auto rows_of = [&](int chunk) { return min(MEM_CHUNK, n - chunk * MEM_CHUNK); };
  const auto decays_of = [&](int chunk, MemDecays& to) {
    return mem_decays(lane < rows_of(chunk) ? g_next : 0.f, lane, reverse, a.in_scale, a.up_scale, to);
  };
  const bool whole_state = a.w.d == DK && (slice + 1) * S::COLS <= cols;

  const int begin = reverse ? c1 - 1 : c0;
  if (c0 < c1) {
    fetch_decays(begin, rows_of(begin));
    if (S::AHEAD) fetch(begin, rows_of(begin));
  }
  srv_floatx4 s[KT] = {};
  const MemPlace<KT> place = {(uint32_t)(4 * g * a.s_row + (col0 + c) * a.s_col), col0 + c < cols ? a.w.d - 4 * g : 0, a.s_row};
  if (!STATES) {
    const int64_t row = mem_begin(a.states, seq, n);
    const float* from = a.starts ? a.starts + (entry * a.heads + head) * a.dk * a.dv : row >= 0 ? a.states.in + (row * a.heads + head) * a.dk * a.dv : nullptr;
    if (from) place.load(from, whole_state, s);
    // a use here: left to the loop, every turn would wait for the loads in flight, the next chunk's
#pragma unroll
    for (int k = 0; k < KT; ++k) asm volatile("" : "+v"(s[k]));
  }
  double grown = 0.0;
  if (c0 < c1 && wave == 0) {
    const double sum = decays_of(begin, decays[0]);
    if (STATES) grown = sum;
  }

  for (int turn = 0; turn < c1 - c0; ++turn) {
    const int chunk = reverse ? c1 - 1 - turn : c0 + turn, rows = rows_of(chunk);
    const int after = reverse ? chunk - 1 : chunk + 1;
    const int64_t t0 = first + (int64_t)chunk * MEM_CHUNK;
    const bool whole = whole_state && rows == MEM_CHUNK;
    asm volatile("" : "+v"(c), "+v"(g));  // places and masks are found anew: kept over the loop they would take registers that spill
    const MemDecays& dl = decays[turn & 1];
    if (!S::AHEAD) fetch(chunk, rows);
    if (turn) __syncthreads();  // the last chunk has been read
    if (!STATES) x_rows.put(xl, rows, a.x.d, whole);
    w_rows.put(wl, rows, a.w.d, whole);
    v_rows.put(vl, rows, cols - slice * S::COLS, whole);
    const bool more = turn + 1 < c1 - c0;
    typename MemFour<T>::type dot[DOTS ? 4 : 1];
    if constexpr (DOTS) {
      const T* const from = static_cast<const T*>(a.dot.p) + head / a.dot.group * a.dot.head + t0 * a.dot.token + col0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        dot[i] = 0;
        if (whole || (16 * i + c < rows && col0 + 4 * g < cols))
          dot[i] = *reinterpret_cast<const typename MemFour<T>::type*>(from + (16 * i * a.dot.token + (c * (uint32_t)a.dot.token + 4 * g)));
      }
    }
    if (more) {
      fetch_decays(after, rows_of(after));  // first: they are used before the rows are
      if (S::AHEAD) fetch(after, rows_of(after));
    }
    __syncthreads();

    srv_floatx4 o[4] = {};
    if constexpr (!STATES) {
      const auto from_state = [&] {  // what the tokens read of the state
#pragma unroll
        for (int k = 0; k < KT; k += 2) {
          op_t part[IN];
          const float x[8] = {s[k][0], s[k][1], s[k][2], s[k][3], s[k + 1][0], s[k + 1][1], s[k + 1][2], s[k + 1][3]};
          mem_split<IN>(x, part);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const T* row = xl + (16 * i + c) * S::XS + 16 * k + 8 * g;
            const op_t y = mem_operand(row, row + 4);
#pragma unroll
            for (int p = IN - 1; p >= 0; --p) o[i] = mem_mma(part[p], y, o[i]);
          }
          if constexpr (S::RESIDENT == 4) __builtin_amdgcn_sched_barrier(0);  // reads that go ahead take registers: spilled ones cost more
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= dl.in[16 * i + c];
        if constexpr (DOTS) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += o[i][r] * srv_widen(dot[i][r]);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (g == 0) meet[wave][16 * i + c] = sum;
          }
        }
      };
      // Pairs first where they have their place beside x: their sums need no registers then that what is read of the state has
      if constexpr (!S::OWN) from_state();
      // pairs: a wavefront has the products of sixteen rows with those, or with every other sixteen of those, that they see
      const int own_rows = wave & 3, j0 = HALVES == 1 ? 0 : wave >> 2;
      op_t second[PAIRS ? S::COLS / 32 : 1];
      if constexpr (PAIRS) {
        const T* const from = static_cast<const T*>(a.dot.p) + head / a.dot.group * a.dot.head + t0 * a.dot.token + slice * S::COLS;
        const uint32_t row = min(16 * own_rows + c, rows - 1) * (uint32_t)a.dot.token;
#pragma unroll
        for (int k = 0; k < S::COLS / 32; ++k) {
          const bool there = slice * S::COLS + 32 * k + 8 * g < cols;
          second[k] = mem_global(from + (row + (there ? 32 * k + 8 * g : 0)), there);
        }
      }
      srv_floatx4 z[4 / HALVES] = {};
#pragma unroll
      for (int k = 0; k < DK / 32; ++k) {
        const T* row = xl + (16 * own_rows + c) * S::XS + 32 * k + mem_place(8 * g);
        const op_t x = mem_operand(row, row + 8);
#pragma unroll
        for (int u = 0; u < 4 / HALVES; ++u) {
          const int j = j0 + HALVES * u;
          if (HALVES == 1 && order * (j - own_rows) > 0) continue;  // (of two wavefronts to sixteen rows both have something to do)
          const T* key = wl + (16 * j + c) * S::XS + 32 * k + 8 * g;
          z[u] = mem_mma(mem_operand(key, key + 4), x, z[u]);
        }
        if constexpr (S::RESIDENT == 4) __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!S::OWN) __syncthreads();  // x has been read
      // Weights: within a sixteen exp(G_i - G_j), a difference at a time; between two of them the product of the way to the end of one, across the
      // sixteens from there to the beginning of the other, and on from there, all at most 1
      const int i = 16 * own_rows + c;
      const float own_since = a.pair_scale * dl.since[i];
      float all = 0.f;  // (with PAIRS) of the row
#pragma unroll
      for (int u = 0; u < 4 / HALVES; ++u) {
        const int j = j0 + HALVES * u;
        float p[4] = {};
        if (j == own_rows) {
          const srv_floatx4 hi = *reinterpret_cast<const srv_floatx4*>(&dl.hi[16 * j + 4 * g]), lo = *reinterpret_cast<const srv_floatx4*>(&dl.lo[16 * j + 4 * g]);
          const float own_hi = dl.hi[i], own_lo = dl.lo[i];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float x = a.pair_scale * z[u][r] * mem_between(own_hi, own_lo, hi[r], lo[r], sign);
            asm volatile("" : "+v"(x));  // (a select, not a branch for every number)
            p[r] = order * (4 * g + r - c) <= 0 ? x : 0.f;
          }
        } else if (order * (j - own_rows) < 0) {
          const srv_floatx4 left = *reinterpret_cast<const srv_floatx4*>(&dl.left[16 * j + 4 * g]);
          const int before = min(j, own_rows), behind = max(j, own_rows);
          const float between = (before < 1 && behind > 1 ? dl.across[1] : 0.f) + (before < 2 && behind > 2 ? dl.across[2] : 0.f);
          const float way = own_since * __builtin_amdgcn_exp2f(between);
#pragma unroll
          for (int r = 0; r < 4; ++r) p[r] = z[u][r] * way * left[r];
        }
        T* const to = pl + i * S::PS + mem_place(16 * j + 4 * g);
        mem_store4(to, p);
        if constexpr (S::PARTS == 2) {
          float rest[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) rest[r] = p[r] - srv_widen(srv_narrow<T>(p[r]));
          mem_store4(to + MEM_CHUNK * S::PS, rest);
        }
        if constexpr (PAIRS) {
          // times the second factor; a pair of one token with itself belongs to no sum
          srv_floatx4 sums = {};
          if (order * (j - own_rows) <= 0) {
            srv_floatx4 y = {};
#pragma unroll
            for (int k = 0; k < S::COLS / 32; ++k) {
              const T* value = vl + (16 * j + c) * S::VS + 32 * k + 8 * g;
              y = mem_mma(mem_operand(value, value + 4), second[k], y);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int e = 16 * j + 4 * g + r;
              float x = p[r] * y[r];
              asm volatile("" : "+v"(x));
              x = order * (e - i) < 0 && max(e, i) < rows ? x : 0.f;
              all += x;
              sums[r] = mem_sixteen(x);
            }
          }
          if (c == 0) *reinterpret_cast<srv_floatx4*>(&meet[own_rows][16 * j + 4 * g]) = sums;
        }
      }
      if constexpr (PAIRS) {
        all += __shfl_xor(all, 16, 64);
        all += __shfl_xor(all, 32, 64);
        if (g == 0) meet[4 + j0][i] = all;
      }
      if constexpr (S::OWN) from_state();
    }
    if (more && wave == ((turn + 1) & (WAVES - 1))) {
      const double sum = decays_of(after, decays[(turn + 1) & 1]);
      if (STATES) grown += sum;
    }
    if constexpr (!STATES) __syncthreads();
    // the values, tokens side by side in a lane
    op_t v[2];
    float finite = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      v[k] = mem_column(vl + 32 * k * S::VS + wave * 16, S::VS, g, c);
      if constexpr (!STATES) finite = mem_finite(v[k], finite);
    }
    if constexpr (!STATES) {
      if constexpr (DOTS)
        if (wave == 0 && lane < rows) {
          float sum = 0.f;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) sum += meet[w][lane];
          a.dots[((int64_t)slice * a.heads + head) * a.m.tokens + t0 + lane] = sum;
        }
      if constexpr (PAIRS)
        if (wave == (turn & (WAVES - 1))) {  // rows are the pairs' earlier tokens, columns the later ones
          double step = meet[4][lane];
          if (HALVES == 2) step += meet[5][lane];
#pragma unroll
          for (int w = 0; w < 4; ++w) step -= meet[w][lane];
          const double sum = mem_sums(step) - step;
          if (lane < rows) a.dots[((int64_t)slice * a.heads + head) * a.m.tokens + t0 + lane] = (float)sum;
        }
      const bool bad = __builtin_amdgcn_ballot_w64(finite != 0.f) != 0;
      op_t clean[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        clean[k] = v[k];
        if (bad) {  // a weight of 0 times NaN would be NaN
          float x[8];
          op_t y[1];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = isfinite(mem_entry(v[k], e)) ? mem_entry(v[k], e) : 0.f;
          mem_split<1>(x, y);
          clean[k] = y[0];
        }
      }
      const auto pairs = [&](int i, int k) {
#pragma unroll
        for (int part = S::PARTS - 1; part >= 0; --part) {
          const T* row = pl + (part * MEM_CHUNK + 16 * i + c) * S::PS + 32 * k + 8 * g;
          o[i] = mem_mma(clean[k], mem_operand(row, row + 4), o[i]);
        }
      };
#pragma unroll
      for (int i = 0; i < 4; ++i) pairs(i, i / 2);
      if (reverse) {
        pairs(0, 1);
        pairs(1, 1);
      } else {
        pairs(2, 0);
        pairs(3, 0);
      }
      if (bad)
        for (int j = 0; j < rows; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float y = srv_widen(vl[j * S::VS + wave * 16 + 4 * g + r]);
              const bool seen = order * (j - (16 * i + c)) <= 0;
              if (seen && !isfinite(y)) o[i][r] += srv_widen(pl[(16 * i + c) * S::PS + mem_place(j & ~3) + (j & 3)]) * y;
            }
      const int64_t out_at = t0 * a.out_token + head * a.out_head + col0;
      const uint32_t mine = c * (uint32_t)a.out_token + 4 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!whole && (16 * i + c >= rows || col0 + 4 * g >= cols)) continue;
        const int64_t to = out_at + 16 * i * a.out_token;
        if (DOTS && a.out_float) mem_out4(static_cast<float*>(a.out) + to + mine, o[i]);
        else mem_out4(static_cast<T*>(a.out) + to + mine, o[i]);
      }
    }
    // the state
    const float fade = dl.whole;
#pragma unroll
    for (int k = 0; k < KT; ++k) s[k] *= fade;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const srv_floatx4 u0 = *reinterpret_cast<const srv_floatx4*>(&dl.up[32 * h + 4 * g]), u1 = *reinterpret_cast<const srv_floatx4*>(&dl.up[32 * h + 16 + 4 * g]);
      op_t up[UP];
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = mem_entry(v[h], e) * (e < 4 ? u0[e & 3] : u1[e & 3]);
      mem_split<UP>(x, up);
#pragma unroll
      for (int k = 0; k < KT; ++k) {
        const op_t w = mem_column(wl + 32 * h * S::XS + 16 * k, S::XS, g, c);
#pragma unroll
        for (int p = UP - 1; p >= 0; --p) s[k] = mem_mma(w, up[p], s[k]);
      }
    }
  }
  float* to = nullptr;
  bool none = false;
  if (STATES) {
    to = a.added + (entry * a.heads + head) * a.dk * a.dv;
    // the wavefronts have the chunks' sums in turn
    double* const all = reinterpret_cast<double*>(&meet[0][0]);
    if (lane == 0) all[wave] = grown;
    __syncthreads();
    if (threadIdx.x == 0 && slice == 0) {
      double sum = 0.0;
      for (int w = 0; w < WAVES; ++w) sum += all[w];
      a.faded[entry * a.heads + head] = exp2f((float)sum);
    }
  } else if (segment == (reverse ? 0 : segments - 1)) {
    const int64_t row = mem_end(a.states, seq);
    if (row >= 0) to = a.states.out + (row * a.heads + head) * a.dk * a.dv;
    none = a.ruled && mem_begin(a.rule, seq, n) < 0;
  }
  if (to) {
    if (whole_state) place.store(to, true, s, none);
    else place.store(to, false, s, none);
  }
}

// The segments' states: what each adds becomes what each finds, four numbers of one head's state to a thread.  The memory bounds it: 67 MB of a gradient's
// states in 12 us.
static __global__ void __launch_bounds__(256) memory_scan_kernel(const MemTwo two) {
  const bool second = blockIdx.x >= two.split;
  const MemArgs& a = two.of[second];
  const uint32_t b = second ? blockIdx.x - two.split : blockIdx.x;
  const int quads = a.dk * a.dv / 4, blocks = (quads + 255) / 256;
  const int head = b / blocks % a.heads, e = (b % blocks * 256 + threadIdx.x) * 4;
  const int64_t seq = b / blocks / a.heads;
  int64_t entry = 0, first;
  int n;
  if (a.m.each) {
    entry = seq * a.m.each;
  } else {
    for (int64_t s = threadIdx.x & 63; s < seq; s += 64) {
      mem_rows(a.m, s, first, n);
      entry += mem_segments(a.m, n);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) entry += __shfl_xor(entry, o, 64);
  }
  if (e >= a.dk * a.dv) return;
  mem_rows(a.m, seq, first, n);
  const int segments = (int)min((int64_t)mem_segments(a.m, n), a.m.entries - entry);  // (fewer only where cu_q does not ascend)
  const int64_t row = mem_begin(a.states, seq, n), size = (int64_t)a.heads * a.dk * a.dv;
  srv_floatx4 now = {};
  if (row >= 0) now = *reinterpret_cast<const srv_floatx4*>(a.states.in + row * size + (int64_t)head * a.dk * a.dv + e);
  float* at = a.added + entry * size + (int64_t)head * a.dk * a.dv + e;
  const float* faded = a.faded + entry * a.heads + head;
  constexpr int AHEAD = 8;  // loads under way
  for (int i = 0; i < segments; i += AHEAD) {
    srv_floatx4 x[AHEAD];
    float f[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i + k < segments) {
        const int seg = a.reverse ? segments - 1 - i - k : i + k;
        x[k] = *reinterpret_cast<const srv_floatx4*>(at + seg * size);
        f[k] = faded[(int64_t)seg * a.heads];
      }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i + k < segments) {
        const int seg = a.reverse ? segments - 1 - i - k : i + k;
        *reinterpret_cast<srv_floatx4*>(at + seg * size) = now;
        now = now * f[k] + x[k];
      }
  }
}

// ---- few tokens ---------------------------------------------------------------------------------------------------------------
// One token after the other, for sequences of few: every state is read once and written once, which is what it takes.  A workgroup has 64 columns of
// a head's state, a thread four of them in every sixteenth row.  64 sequences of 32 heads of 128 x 128: 49 us a call for 268 MB, 5.5 TB/s; the
// memory bounds it.

constexpr int MEM_STEP_ROWS = 16;

template <typename T, int DK>
__global__ void __launch_bounds__(256) memory_step_kernel(const MemArgs a) {
  constexpr int ROWS = DK / MEM_STEP_ROWS;
  __shared__ alignas(16) float xl[DK], wl[DK], meet[4][64];
  const int tid = threadIdx.x, col = tid % 16 * 4, r0 = tid / 16;
  const int slice = blockIdx.x % a.slices, head = blockIdx.x / a.slices % a.heads, e = slice * 64 + col;
  const int64_t seq = blockIdx.x / a.slices / a.heads;
  int64_t first;
  int n;
  mem_rows(a.m, seq, first, n);
  const int64_t from = mem_begin(a.states, seq, n), to = mem_end(a.states, seq);
  const bool mine = e < a.dv;
  srv_floatx4 s[ROWS] = {};
  if (from >= 0 && mine) {
    const float* p = a.states.in + (from * a.heads + head) * a.dk * a.dv + e;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (r0 + 16 * i < a.dk) s[i] = *reinterpret_cast<const srv_floatx4*>(p + (int64_t)(r0 + 16 * i) * a.dv);
  }
  const T* xp = static_cast<const T*>(a.x.p) + head / a.x.group * a.x.head;
  const T* wp = static_cast<const T*>(a.w.p) + head / a.w.group * a.w.head;
  const T* vp = static_cast<const T*>(a.v.p) + head * a.v.head + e;
  for (int t = 0; t < n; ++t) {
    const int64_t at = first + t;
    __syncthreads();
    if (tid < DK) {
      xl[tid] = tid < a.dk ? srv_widen(xp[at * a.x.token + tid]) : 0.f;
      wl[tid] = tid < a.dk ? srv_widen(wp[at * a.w.token + tid]) : 0.f;
    }
    float v[4] = {};
    if (mine)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = srv_widen(vp[at * a.v.token + k]);
    const float fade = expf(mem_decay(a.log_decay[at * a.g_token + head * a.g_head]));
    __syncthreads();
    srv_floatx4 o = {};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float w = wl[r0 + 16 * i], x = xl[r0 + 16 * i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[i][k] = s[i][k] * fade + w * v[k];
        o[k] += x * s[i][k];
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      o[k] += __shfl_xor(o[k], 16, 64);
      o[k] += __shfl_xor(o[k], 32, 64);
    }
    if ((tid & 63) < 16) *reinterpret_cast<srv_floatx4*>(&meet[tid >> 6][col]) = o;
    __syncthreads();
    if (tid < 64 && slice * 64 + tid < a.dv) {
      const float y = a.in_scale * ((meet[0][tid] + meet[1][tid]) + (meet[2][tid] + meet[3][tid]));
      static_cast<T*>(a.out)[at * a.out_token + head * a.out_head + slice * 64 + tid] = srv_narrow<T>(y);
    }
  }
  if (to >= 0 && mine) {
    float* p = a.states.out + (to * a.heads + head) * a.dk * a.dv + e;
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
      if (r0 + 16 * i < a.dk) *reinterpret_cast<srv_floatx4*>(p + (int64_t)(r0 + 16 * i) * a.dv) = s[i];
  }
}

}  // namespace ttc
