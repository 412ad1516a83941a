// Attention over the cache in 4 bits (ttc_attention): out = softmax(scale q K^T) V, one pass over the context with the running maximum
// and sum of the softmax.
//
// A row is one new token of one query head; the rows of a tile read the same cache head.  Both products run on the matrix cores with the
// rows as columns: S^T = K Q^T (16 tokens x 16 rows) leaves in each lane four tokens' scores of one row, and these are what the
// lane has to hold for O^T = V^T P^T, whose sum runs over the tokens, if the tokens of two such tiles are taken in the order in which the
// lanes hold them.  So the weights never move between lanes, maxima and sums are the lane's own but for one exchange among four lanes,
// and rescaling is a product of the lane's own numbers.  The four wavefronts of a workgroup take 64 tokens each in turn and join their sums
// at the end: with few rows it is the context that has to be divided.
//
// What bounds it: 4 sequences of 131072 tokens (8 cache heads of 128, 4 query heads each, bfloat16) are read in 95 us, 6.0 TB/s, where a
// kernel that only reads reaches 6.7 to 7.2; 64 sequences of 257 to 16384 tokens in 118 us, 5.0 TB/s, the rest being the beginnings and
// joins of a workgroup's two items or three.  24 sequences of up to 4099 tokens in float32 (16 heads of 64) take 32 us for 10.7 us of
// bytes: four units a workgroup, and products of three parts.  One sequence of 4099 tokens takes 12 us: a chain of waits (lengths,
// page numbers, codes, join) for 0.9 us of bytes.
//
// Roundings: scores, statistics and sums are float32.  With bfloat16 rows a weight is rounded to bfloat16 for its product with the values, one
// product instead of three and the operand type that the queries came in; the sum that divides is of the unrounded weights.  That moves an
// entry of the result by 2^-8 of sum weight |value| at most, as much as its own rounding to bfloat16 does.  Rows of float32 round nothing: a number is
// the sum of three bfloat16 parts, which hold its 24 bits.
#pragma once
#include "ttc_attention_plan.hpp"
#include "ttc_serve.hpp"

namespace ttc {

// What nothing writes during the launch: read through the scalar cache where all lanes want the same
typedef __attribute__((address_space(4))) int32_t att_const_int;

// The row tile of a workgroup: its sequence's numbers and this lane's row
struct AttTile {
  int len;          // tokens in the cache
  int rows;         // rows of the sequence
  int64_t first_q;  // row of q of its first new token
  int first, last;  // tokens that the lane's row sees: first .. last (none where last < first)
  int lo, hi;       // all that the tile's rows see lies in lo .. hi-1
  int all_lo, all_hi;  // and every one of them sees all of all_lo .. all_hi-1
  int real;         // rows of the tile
};

template <int ROWS = ATT_ROWS>
__device__ __forceinline__ AttTile att_tile(const AttentionArgs& p, int64_t seq, int tile, int row) {
  const ttc_attention_t& a = p.a;
  AttTile t;
  int64_t q0 = seq, q1 = seq + 1;
  if (a.cu_q) {
    const att_const_int* const cu = (const att_const_int*)a.cu_q;
    q0 = cu[seq];
    q1 = cu[seq + 1];
  }
  q0 = q0 < 0 ? 0 : q0;
  q1 = q1 > a.tokens ? a.tokens : q1;
  int64_t m = q1 - q0;
  const int64_t all = m;  // (positions count every new token, also those behind max_q)
  m = m < 0 ? 0 : m > a.max_q ? a.max_q : m;
  const int len = ((const att_const_int*)a.kv_len)[seq];
  t.len = len < 0 ? 0 : len > a.max_kv ? a.max_kv : len;
  t.rows = (int)m * p.group;
  t.first_q = q0;
  const int r = tile * ROWS + row;
  const int r1 = min(t.rows, (tile + 1) * ROWS) - 1;  // last row of the tile
  const int shift = t.len - (int)all;                     // token number of the first new one
  if (a.causal) {
    t.last = min(shift + r / p.group, t.len - 1);
    t.first = a.window ? max(t.last - a.window + 1, 0) : 0;
    t.hi = min(shift + r1 / p.group, t.len - 1) + 1;
    const int first = min(shift + tile * ROWS / p.group, t.len - 1);  // what the first row sees last
    t.lo = a.window ? max(first - a.window + 1, 0) : 0;
    t.all_lo = a.window ? max(t.hi - a.window, 0) : 0;
    t.all_hi = first + 1;
  } else {
    t.last = t.len - 1;
    t.first = 0;
    t.hi = t.all_hi = t.len;
    t.lo = t.all_lo = 0;
  }
  t.real = max(r1 - tile * ROWS + 1, 0);
  if (r >= t.rows) t.last = -1;
  if (!t.real) t.hi = 0;
  t.lo = t.lo / ATT_STEP * ATT_STEP;
  return t;
}

// units of 256 tokens of one item; one for rows that see nothing, whose results somebody has to write
__device__ __forceinline__ uint32_t att_units(const AttTile& t) {
  return t.hi > t.lo ? (uint32_t)(t.hi - t.lo + ATT_UNIT - 1) / ATT_UNIT : t.real ? 1 : 0;
}

// The entries (sequence, row tile) in their order, each of `heads` items of its number of units: every wavefront adds them up for
// itself, a run of entries to a lane.
struct AttShares {
  uint32_t total;   // units of all items
  uint32_t before;  // of the entries before this lane's run
  uint32_t own;     // of this lane's run
  int first, last;  // the run: first .. last-1
  __device__ __forceinline__ explicit AttShares(const AttentionArgs& p) {
    const int lane = threadIdx.x & 63, run = (p.entries + 63) / 64;
    first = min(lane * run, p.entries);
    last = min(first + run, p.entries);
    own = 0;
    for (int i = first; i < last; ++i) own += att_units(att_tile(p, i / p.row_tiles, i % p.row_tiles, 0));
    own *= p.a.cache.heads;
    uint32_t sum = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(sum, o, 64);
      sum += lane >= o ? x : 0;
    }
    total = __builtin_amdgcn_readlane(sum, 63);
    before = sum - own;
  }
  // the entry that unit u of all is of (u < total), and the entry's units before it
  __device__ __forceinline__ int find(const AttentionArgs& p, uint32_t u, uint32_t& rest) const {
    const int lane = __builtin_ctzll(__builtin_amdgcn_ballot_w64(u >= before && u < before + own));
    uint32_t at = __builtin_amdgcn_readlane(before, lane);
    if (p.entries <= 64) {  // a run is one entry
      rest = u - at;
      return lane;
    }
    for (int i = __builtin_amdgcn_readlane(first, lane);; ++i) {
      const uint32_t n = __builtin_amdgcn_readfirstlane(att_units(att_tile(p, i / p.row_tiles, i % p.row_tiles, 0))) * p.a.cache.heads;
      if (u < at + n || i + 1 >= p.entries) {
        rest = u - at;
        return i;
      }
      at += n;
    }
  }
};

// A float32 number as the sum of TERMS bfloat16 ones: one, rounded, or three that give every bit
template <int TERMS>
__device__ __forceinline__ void att_split(float x, __bf16 (&t)[TERMS]) {
#pragma unroll
  for (int i = 0; i < TERMS; ++i) {
    t[i] = static_cast<__bf16>(x);
    x -= static_cast<float>(t[i]);
  }
}

// Eight codes (a word) to eight bfloat16 numbers, exactly: a code has two significant bits, the scale is a power of two
__device__ __forceinline__ srv_bf16x8 att_widen(uint32_t code, float scale) {
  const srv_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1),
                   c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
  return srv_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 128 in every byte above 252: the exponents of blocks that are NaN
__device__ __forceinline__ uint32_t att_nan_bytes(uint32_t x) { return x & ((x & 0x7f7f7f7fu) + (0x7f - (KV_LARGEST & 0x7f)) * 0x01010101u) & 0x80808080u; }

// Codes of a wavefront's step, which nobody else reads soon: past the caches' replacement, 97 us a call instead of 110 over 4 x 131072 tokens,
// 125 instead of 132 over 64 sequences of 257 to 16384 (d = 128).  With heads of 256 a lane's 32 bytes take two reads of the same lines,
// and the second may miss (16 x 4096 tokens 27.6 us instead of 26.7).
template <int D, typename W>
__device__ __forceinline__ W att_stream(const W* p) {
  if constexpr (D <= 128) return __builtin_nontemporal_load(p);
  else return *p;
}

// What a workgroup reads the cache with, the same for all of its lanes
struct AttSource {
  const unsigned char* cache;  // the workgroup's head of page 0
  const att_const_int* pages;  // the sequence's
  int64_t page_stride;
  uint32_t page_count;
  int page_tokens, log_page, end;
  __device__ __forceinline__ AttSource(const AttentionArgs& p, int64_t seq, int head, int end_) : end(end_) {
    const ttc_kv_cache_t& c = p.a.cache;
    const int64_t bytes = (int64_t)c.page * (c.d + c.d / 16);
    cache = static_cast<const unsigned char*>(c.data) + head * bytes;
    pages = (const att_const_int*)(p.a.block_table + seq * p.a.table_stride);
    page_stride = c.heads * bytes;
    page_count = (uint32_t)min(c.pages, (int64_t)INT32_MAX);
    page_tokens = c.page;
    log_page = __builtin_ctz(c.page);
  }
  // What the table says of the four sixteens from token n0 on, not yet looked at (whoever looks waits for it)
  __device__ __forceinline__ void look_up(int n0, int (&page)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) page[i] = pages[min(n0 + 16 * i, end - 1) >> log_page];
  }
  // bit i is set if the page of sixteen i is in the cache
  __device__ __forceinline__ int there(int n0, const int (&page)[4]) const {
    int bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= n0 + 16 * i < end && (uint32_t)page[i] < page_count ? 1 << i : 0;
    return bits;
  }
  __device__ __forceinline__ const unsigned char* base(int page) const { return cache + ((uint32_t)page < page_count ? page : 0) * page_stride; }
};

// A wavefront's share of one step of 64 tokens, as it lies in the cache: lane (c, g) has the entries g*D/4 .. of the keys of token c of each
// sixteen, and entries c*D/16 .. of the values of tokens 4g .. 4g+3.  `there` as in AttSource.
template <int D>
struct AttKeys {
  typedef KvParts<D> P;
  typedef uint32_t word_t __attribute__((ext_vector_type(D / 32)));
  word_t code[4];
  uint32_t exp[4];
  int there;
  __device__ __forceinline__ void load(const AttSource& s, const int (&page)[4], int n0, int c, int g) {
    there = s.there(n0, page);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned char* base = s.base(page[i]);
      const uint32_t token = ((n0 + 16 * i) & (s.page_tokens - 1)) + c;
      code[i] = att_stream<D>(reinterpret_cast<const word_t*>(base + (token * P::TOKEN + g * (D / 8))));
      const uint32_t at = P::key_exps(s.page_tokens) + token * P::BLOCKS;
      exp[i] = D == 256 ? *reinterpret_cast<const unsigned short*>(base + (at + 2 * g)) : base[at + (D == 64 ? g / 2 : g)];
    }
  }
};
template <int D>
struct AttValues {
  typedef KvParts<D> P;
  typedef uint32_t word_t __attribute__((ext_vector_type(D / 32)));
  word_t code[4];
  uint32_t exp[4];
  __device__ __forceinline__ void load(const AttSource& s, const int (&page)[4], int n0, int c, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned char* base = s.base(page[i]);
      const uint32_t four = ((n0 + 16 * i) & (s.page_tokens - 1)) / 4 + g;
      code[i] = att_stream<D>(reinterpret_cast<const word_t*>(base + (P::values(s.page_tokens) + (four * 16 + c) * (4 * P::LANE))));
      exp[i] = *reinterpret_cast<const uint32_t*>(base + (P::value_exps(s.page_tokens) + (four * P::BLOCKS + c * (D / 16) / 32) * 4));
    }
  }
};

// entries e, e+1 of token k of the four whose codes a lane holds: E/2 bytes a token
template <int E, typename W>
__device__ __forceinline__ srv_bf16x2 att_value_pair(const W& code, int k, int e, float scale) {
  const int byte = k * (E / 2) + e / 2;
  const uint32_t word = code[byte / 4];
  switch (byte % 4) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3);
  }
}

// A workgroup had some of an item's units: its result goes to a slot of the workspace, and whoever finds that all have arrived joins them, in
// the order of the units, so that equal calls give equal bits.  True for the threads that then hold entries e0 .. of row `row` of the whole.
//
// Arrival is a mark in the slot, of 64 bits that no earlier contents of the workspace have but by chance (1 in 2^64); the caller need
// not clear anything.  Every workgroup sets its own mark and then looks at the others', so the last one sees all; two may, and then both
// write the same.  The marks are taken away again, for a captured launch comes back with the same one.  Nobody waits for another workgroup.
// The workgroups may be on different XCDs, whose caches do not see each other's lines: results and marks go past them, in stores and loads
// of device scope.  Each wavefront waits for its stores, the workgroup for its wavefronts, and only then the mark is set.  That order rests on
// the hardware, whose memory counter (vmcnt) says when a store of device scope has arrived, not on the language, to which relaxed accesses
// of different addresses have none.
// Fences of device scope instead write back and empty whole caches: a call over 4 x 131072 tokens took 282 us with them.  A count of
// arrivals, which all workgroups of an item change one after the other, took 26 us where the marks take 13 (17 workgroups, 4099 tokens).
__device__ __forceinline__ void att_put2(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void att_get2(const float* p, float& a, float& b) {
  const unsigned long long x = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  a = __uint_as_float((uint32_t)x);
  b = __uint_as_float((uint32_t)(x >> 32));
}
template <int D>
__device__ __forceinline__ bool att_join(const AttentionArgs& p, const AttTile& t, uint32_t first_unit, uint32_t units, uint32_t total, uint32_t used,
                                         uint32_t slot, int& row, int e0, float& mm, float& ll, float (&sum)[D / 16], float* part_o,
                                         float* part_m, int* joins) {
  constexpr int E = D / 16;
  if (row < t.real) {
    float* stat = p.part_stat + ((int64_t)slot * ATT_ROWS + row) * 2;
    float* out = p.part_out + ((int64_t)slot * ATT_ROWS + row) * D + e0;
    if (threadIdx.x % 16 == 0) att_put2(stat, mm, ll);
#pragma unroll
    for (int e = 0; e < E; e += 2) att_put2(out + e, sum[e], sum[e + 1]);
  }
  // workgroup w has the units from total * w / used on; the item's first may have begun with another item
  const uint32_t w0 = (uint32_t)(((uint64_t)(first_unit + 1) * used - 1) / total);
  const uint32_t parts = (uint32_t)(((uint64_t)(first_unit + units) * used - 1) / total) - w0 + 1;
  const uint32_t slot0 = (uint32_t)((uint64_t)total * w0 / used) < first_unit ? 1 : 0;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x < 64) {
    if (threadIdx.x == 0) (void)__hip_atomic_exchange(p.marks + slot, p.mark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bool all = true;
    for (uint32_t s = threadIdx.x; s < parts; s += 64)
      all &= __hip_atomic_load(p.marks + 2 * ((int64_t)w0 + s) + (s == 0 ? slot0 : 0), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == p.mark;
    const bool arrived = __builtin_amdgcn_ballot_w64(!all) == 0;
    if (threadIdx.x == 0) *joins = arrived;
  }
  __syncthreads();
  if (!*joins) return false;
  asm volatile("" ::: "memory");
  for (uint32_t s = threadIdx.x; s < parts; s += 64 * ATT_WAVES)
    __hip_atomic_store(p.marks + 2 * ((int64_t)w0 + s) + (s == 0 ? slot0 : 0), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // 16 threads to a row, and as many groups of them to the same row as there are rows to spare; each group takes every so many-th part
  int rows = 1;
  while (rows < t.real) rows <<= 1;
  const int group = threadIdx.x / 16, groups = ATT_ROWS / rows, first = group / rows;
  row = group % rows;
  mm = -INFINITY;
  ll = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  if (row < t.real) {
    // four parts' loads under way before the first is used
    for (uint32_t s0 = first; s0 < parts; s0 += 4 * groups) {
      float ms[4], ls[4], x[4][E];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t s = s0 + k * groups < parts ? s0 + k * groups : s0;
        const int64_t at = (2 * ((int64_t)w0 + s) + (s == 0 ? slot0 : 0)) * ATT_ROWS + row;
        att_get2(p.part_stat + at * 2, ms[k], ls[k]);
#pragma unroll
        for (int e = 0; e < E; e += 2) att_get2(p.part_out + at * D + e0 + e, x[k][e], x[k][e + 1]);
      }
      float top = mm;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ms[k] = s0 + k * groups < parts ? ms[k] : -INFINITY;
        top = fmaxf(top, ms[k]);
      }
      const float zero = top == -INFINITY ? 0.f : top, f = __builtin_amdgcn_exp2f(mm - zero);
      mm = top;
      ll *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] *= f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (s0 + k * groups >= parts) break;
        const float h = __builtin_amdgcn_exp2f(ms[k] - zero);
        ll += h * ls[k];
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += h * x[k][e];
      }
    }
  }
  if (groups == 1) return row < t.real;
  float* const o = part_o + group * (D + 4) + e0;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = sum[e];
  if (threadIdx.x % 16 == 0) {
    part_m[2 * group] = mm;
    part_m[2 * group + 1] = ll;
  }
  __syncthreads();
  if (first || row >= t.real) return false;
  for (int i = 1; i < groups; ++i) mm = fmaxf(mm, part_m[2 * (i * rows + row)]);
  const float zero = mm == -INFINITY ? 0.f : mm;
  ll = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.f;
  for (int i = 0; i < groups; ++i) {
    const int at = i * rows + row;
    const float f = __builtin_amdgcn_exp2f(part_m[2 * at] - zero);
    ll += f * part_m[2 * at + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += f * part_o[at * (D + 4) + e0 + e];
  }
  return true;
}

template <typename T, int D>
__global__ void __launch_bounds__(64 * ATT_WAVES, att_resident(D)) attention_kernel(const AttentionArgs p) {
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int TERMS = BF16 ? 1 : 3;   // bfloat16 parts of a query and of a weight
  constexpr int KS = D / 32;            // products of 32 entries that a score takes
  constexpr int E = D / 16;             // entries of a value that a lane holds
  const ttc_attention_t& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
  __shared__ float part_o[ATT_WAVES][ATT_ROWS][D + 4];
  __shared__ float part_m[ATT_WAVES][ATT_ROWS], part_l[ATT_WAVES][ATT_ROWS];
  __shared__ int joins;

  // The workgroup's units: unit .. stop-1 of all; of entry `entry` from its unit `rest` on (the entry's heads one after the other)
  uint32_t unit = 0, stop = 1, rest = 0, total = 0, used = 0;
  int entry = 0, head = 0;
  if (p.shared) {
    const AttShares all(p);
    total = all.total;
    used = min(total, gridDim.x);  // workgroups with any unit
    if (blockIdx.x >= used) return;
    unit = (uint32_t)((uint64_t)total * blockIdx.x / used);
    stop = (uint32_t)((uint64_t)total * (blockIdx.x + 1) / used);
    entry = all.find(p, unit, rest);
  } else {
    entry = (int)(blockIdx.x / a.cache.heads);
    head = (int)(blockIdx.x % a.cache.heads);
  }
  bool first_item = true;
  while (unit < stop) {
    const int64_t seq = entry / p.row_tiles;
    const int tile = entry % p.row_tiles;
    const AttTile t = att_tile(p, seq, tile, c);
    const uint32_t units = __builtin_amdgcn_readfirstlane(att_units(t));
    uint32_t take = units, from = 0;
    if (p.shared) {
      if (rest >= units * a.cache.heads) {  // the next entry (the first one found is not done yet)
        ++entry;
        rest = 0;
        continue;
      }
      head = (int)(rest / units);
      from = rest % units;
      take = min(units - from, stop - unit);
    }
    const int begin = t.lo + (int)from * ATT_UNIT, end = min(t.hi, begin + (int)take * ATT_UNIT);

    // page numbers, queries and the first step's codes are on their way together
    const AttSource src(p, seq, head, end);
    constexpr int STRIDE = ATT_STEP * ATT_WAVES;
    int page[4], n0 = begin + wave * ATT_STEP;
    if (n0 < end) src.look_up(n0, page);

    // the lane's share of its row: entries g*D/4 .. of every part
    srv_bf16x8 q[TERMS][KS];
    float query[BF16 ? 1 : KS][8];
    {
      const int r = tile * ATT_ROWS + c;
      const bool real = r < t.rows;
      const int64_t at = real ? (t.first_q + r / p.group) * a.q_token + (int64_t)(head * p.group + r % p.group) * a.q_head : 0;
      const T* x = static_cast<const T*>(a.q) + at + g * (D / 4);
      const bool vec = (uint64_t)a.q % 16 == 0 && (a.q_token | a.q_head) % (16 / (int)sizeof(T)) == 0;
  #pragma unroll
      for (int s = 0; s < KS; ++s) {
        if constexpr (BF16) {
          q[0][s] = srv_bf16x8{};
          if (real) q[0][s] = srv_ld8_bf16(x + 8 * s, vec);
        } else {
  #pragma unroll
          for (int i = 0; i < 8; ++i) query[s][i] = 0.f;
          if (real) srv_ld8(x + 8 * s, vec, query[s]);
        }
      }
    }
    srv_floatx4 o[E] = {};
    float m = -INFINITY, l = 0.f;
    const float to_log2 = a.scale * 1.44269504088896340736f;
    // Keys and values of the next step are read into the registers that this step has just done with, and the page numbers of the step
    // after it: the reads are under way during the other product and the softmax, and while other wavefronts of the SIMD work.
    AttKeys<D> keys;
    AttValues<D> values;
    if (n0 < end) {
      keys.load(src, page, n0, c, g);
      values.load(src, page, n0, c, g);
      src.look_up(n0 + STRIDE, page);
    }
    if constexpr (!BF16) {
  #pragma unroll
      for (int s = 0; s < KS; ++s)
  #pragma unroll
        for (int i = 0; i < 8; ++i) {
          __bf16 part[TERMS];
          att_split<TERMS>(query[s][i], part);
  #pragma unroll
          for (int k = 0; k < TERMS; ++k) q[k][s][i] = part[k];
        }
    }
    for (; n0 < end; n0 += STRIDE) {
      const bool more = n0 + STRIDE < end;
      const int there = keys.there;
      // scores: S^T = K Q^T, sixteen tokens at a time
      srv_floatx4 z[4];
  #pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i] = srv_floatx4{};
  #pragma unroll
        for (int k = 0; k < KS; ++k) {
          const srv_bf16x8 key = att_widen(keys.code[i][k], srv_scale_or_nan((keys.exp[i] >> (D == 256 ? 8 * (k / 4) : 0)) & 255));
  #pragma unroll
          for (int x = TERMS - 1; x >= 0; --x) z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[x][k], z[i], 0, 0, 0);
        }
      }
      if (more) keys.load(src, page, n0 + STRIDE, c, g);
      if (n0 < t.all_lo || n0 + ATT_STEP > t.all_hi || there != 15) {
  #pragma unroll
        for (int i = 0; i < 4; ++i)
  #pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int n = n0 + 16 * i + 4 * g + j;
            z[i][j] = (there >> i & 1) && n >= t.first && n <= t.last ? z[i][j] * to_log2 : -INFINITY;
          }
      } else {
  #pragma unroll
        for (int i = 0; i < 4; ++i) z[i] *= to_log2;
      }
      // The maximum that weights are relative to moves only when a score passes it by 8 (weights stay below 2^8, which costs float32 sums
      // nothing): most steps need no exchange between lanes and no rescaling.
      float top = -INFINITY;
  #pragma unroll
      for (int i = 0; i < 4; ++i)
  #pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, z[i][j]);
      if (__builtin_amdgcn_ballot_w64(top > m + 8.f)) {
        top = fmaxf(m, top);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));  // (a row that has seen nothing yet)
        m = top;
        l *= shrink;
  #pragma unroll
        for (int i = 0; i < E; ++i) o[i] *= shrink;
      }
      const float zero = m == -INFINITY ? 0.f : m;
  #pragma unroll
      for (int i = 0; i < 4; ++i)
  #pragma unroll
        for (int j = 0; j < 4; ++j) {
          z[i][j] = __builtin_amdgcn_exp2f(z[i][j] - zero);
          l += z[i][j];
        }
      // O^T += V^T P^T, 32 tokens at a time: lane (c, g) has tokens 4g .. 4g+3 of two sixteens
  #pragma unroll
      for (int h = 0; h < 2; ++h) {
        srv_bf16x8 w[TERMS];
  #pragma unroll
        for (int k = 0; k < 8; ++k) {
          __bf16 part[TERMS];
          att_split<TERMS>(z[2 * h + k / 4][k % 4], part);
  #pragma unroll
          for (int x = 0; x < TERMS; ++x) w[x][k] = part[x];
        }
        uint32_t exps[2] = {values.exp[2 * h], values.exp[2 * h + 1]};
        // A weight of 0 takes out any number, but neither NaN nor infinity, and what lies behind a sequence's end may be any bytes.  Blocks
        // whose exponents stand for NaN are rare: they are read as (finite) numbers, and what the rows that see them get is made NaN by a
        // product of its own.
        const uint32_t nan0 = att_nan_bytes(exps[0]), nan1 = att_nan_bytes(exps[1]);
        if (__builtin_amdgcn_ballot_w64((nan0 | nan1) != 0)) {
          srv_bf16x8 bad, seen;
  #pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int i = 2 * h + k / 4, n = n0 + 16 * i + 4 * g + k % 4;
            bad[k] = static_cast<__bf16>((k < 4 ? nan0 : nan1) >> (8 * (k % 4)) & 128 ? 1.f : 0.f);
            seen[k] = static_cast<__bf16>((there >> i & 1) && n >= t.first && n <= t.last ? 1.f : 0.f);
          }
          const srv_floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, seen, srv_floatx4{}, 0, 0, 0);
  #pragma unroll
          for (int j = 0; j < 4; ++j)
  #pragma unroll
            for (int e = 0; e < E; ++e) o[e][j] = hit[j] > 0.f ? __builtin_nanf("") : o[e][j];
          exps[0] ^= nan0;
          exps[1] ^= nan1;
        }
  #pragma unroll
        for (int e = 0; e < E; e += 2) {
          srv_bf16x8 v0, v1;
  #pragma unroll
          for (int k = 0; k < 8; ++k) {
            const srv_bf16x2 two = att_value_pair<E>(values.code[2 * h + k / 4], k % 4, e, srv_scale((exps[k / 4] >> (8 * (k % 4))) & 255));
            v0[k] = two[0];
            v1[k] = two[1];
          }
  #pragma unroll
          for (int x = TERMS - 1; x >= 0; --x) {
            o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w[x], o[e], 0, 0, 0);
            o[e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w[x], o[e + 1], 0, 0, 0);
          }
        }
      }
      if (more) {
        values.load(src, page, n0 + STRIDE, c, g);
        src.look_up(n0 + 2 * STRIDE, page);
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // the wavefronts' results join: lane (c, g) holds entries (4g + j)*E + e of row c
  #pragma unroll
    for (int j = 0; j < 4; ++j)
  #pragma unroll
      for (int e = 0; e < E; ++e) part_o[wave][c][(4 * g + j) * E + e] = o[e][j];
    if (g == 0) {
      part_m[wave][c] = m;
      part_l[wave][c] = l;
    }
    __syncthreads();
    int row = threadIdx.x / 16;
    const int e0 = (threadIdx.x % 16) * E;
    float mm = -INFINITY, ll = 0.f, sum[E] = {};
  #pragma unroll
    for (int w = 0; w < ATT_WAVES; ++w) mm = fmaxf(mm, part_m[w][row]);
    const float zero = mm == -INFINITY ? 0.f : mm;
  #pragma unroll
    for (int w = 0; w < ATT_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(part_m[w][row] - zero);
      ll += f * part_l[w][row];
  #pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += f * part_o[w][row][e0 + e];
    }
    bool writes = row < t.real;
    if (take < units) writes = att_join<D>(p, t, unit - from, units, total, used, 2 * blockIdx.x + (first_item ? 0 : 1), row, e0,
                                           mm, ll, sum, &part_o[0][0][0], &part_m[0][0], &joins);
    if (writes) {
      const float f = ll > 0.f || ll != ll ? 1.f / ll : 0.f;
      const int r = tile * ATT_ROWS + row;
      const int64_t token = t.first_q + r / p.group;
      const int h = head * p.group + r % p.group;
      T* y = static_cast<T*>(a.out) + token * a.out_token + (int64_t)h * a.out_head + e0;
  #pragma unroll
      for (int e = 0; e < E; ++e) sum[e] *= f;
      srv_st(y, (uint64_t)a.out % 16 == 0 && (a.out_token | a.out_head) % (16 / (int)sizeof(T)) == 0, sum);
      if (a.lse && threadIdx.x % 16 == 0) a.lse[token * a.heads_q + h] = (mm + __builtin_log2f(ll)) * 0.69314718055994530942f;
    }
    if (!p.shared) return;
    unit += take;
    rest += take;
    first_item = false;
    __syncthreads();  // before the next item's results
  }
}

}  // namespace ttc
