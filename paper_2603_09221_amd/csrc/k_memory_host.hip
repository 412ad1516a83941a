// Plans and launches of linear attention, and the kernels that do not depend on the heads' size.
#include "ttc_memory_backward.hpp"
#include "ttc_memory_launch.hpp"

namespace ttc {

template <> hipError_t launch_memory_chunks<64>(const MemTwo&, bool, int, int, uint32_t, hipStream_t);
template <> hipError_t launch_memory_chunks<128>(const MemTwo&, bool, int, int, uint32_t, hipStream_t);
template <> hipError_t launch_memory_chunks<256>(const MemTwo&, bool, int, int, uint32_t, hipStream_t);
template <> hipError_t launch_memory_step<64>(const MemArgs&, bool, uint32_t, hipStream_t);
template <> hipError_t launch_memory_step<128>(const MemArgs&, bool, uint32_t, hipStream_t);
template <> hipError_t launch_memory_step<256>(const MemArgs&, bool, uint32_t, hipStream_t);

namespace {

// Tokens of a sequence up to which memory_step_kernel takes it.  256 sequences, 16 heads of 128 x 128, step / chunks in us: bfloat16 with 4 tokens 107 / 133,
// 6: 124 / 140, 8: 143 / 137; float32, whose chunks are matrix instructions of an eighth of the rate, with 8: 140 / 319, 16: 202 / 323.  64 sequences, 32 heads
// of 64: 21 / 32 with 6 and 36 / 60 with 16.
int step_most(bool bf16) { return bf16 ? 6 : 16; }

// Columns of a workgroup, and workgroups to the columns of a state: 128, for rows and pairs' products are shared by more (16384 tokens of 32 heads 228 us, with
// 64 columns 289).  float32 rows of more than 128 entries leave LDS room for 64.
int columns_of(int rows, int cols, bool bf16) { return cols > 64 && (bf16 || rows <= 128) ? 128 : 64; }
int slices_of(int rows, int cols, bool bf16) { return (cols + columns_of(rows, cols, bf16) - 1) / columns_of(rows, cols, bf16); }

// Blocks of heads: one where there are segments for the XCDs to take in turn, two for each, else the fewest that make as many (512 tokens of 64 heads: 39 us,
// with one block 50; 64 tokens: 14.7 and 17.1)
int blocks_of(int64_t entries, int heads) {
  int n = 1;
  while (n < heads && (entries * n < 16 || heads % n)) ++n;
  return n;
}
// Sequences in segments.  A sequence has places for as many as the longest has, or, where that takes more than `wider` times as many, sequences have what they
// need, which every workgroup has to add up (gradients of 8192 times 72 tokens, 8 heads: 14.7 ms so).
MemSequences sequences_of(const ttc_linear_attention_t& a, int segment, int wider) {
  const int64_t rows = (int64_t)segment * MEM_CHUNK, longest = a.max_q < a.tokens ? a.max_q : a.tokens;
  const int64_t each = longest <= rows ? 1 : (longest + rows - 1) / rows, tight = each == 1 ? a.sequences : a.sequences + a.tokens / rows;
  MemSequences m = {a.sequences, a.tokens, a.cu_q, a.max_q, segment, tight, 0, 1};
  if (each == 1 || ((double)a.sequences * each <= (double)tight * wider && (double)a.sequences * each * a.heads < 8388608.)) {  // (threads of a launch: 2^32)
    m.entries = a.sequences * each;
    m.each = (int32_t)each;
  }
  m.blocks = blocks_of(m.entries, a.heads);
  return m;
}
// Workgroups of mem_deal
uint32_t dealt(const MemSequences& m, int heads, int per_head) {
  return (uint32_t)((m.entries * m.blocks + 7) / 8 * 8 * (heads / m.blocks) * per_head);
}

// Chunks of a segment: all of a sequence where sequences, heads and slices give every compute unit the two workgroups that LDS has room for, else the
// fewest with which there are no more than two a unit, for a third waits until another is done.  Of sequences of different lengths (the host knows how many
// tokens they have) half a segment each is taken to be left over.  One sequence of 16384 tokens, 32 heads, bfloat16: 228 us; 269, 252 and 247 with one, three
// and four workgroups a unit; twelve of up to 1500 tokens, 16 heads, float32: 104; 153, 115, 113; gradients of four times 2048 tokens, 16 heads: 230; 301,
// 262, 244.  At least two chunks, for a state is as much to write and to read as a chunk's rows: gradients of three of up to 1999 tokens, 8 heads, float32:
// 139 us, as with one; 171 and 153 with three and four.
int segment_of(const ttc_linear_attention_t& a, int slices, int cus) {
  const int64_t longest = a.max_q < a.tokens ? a.max_q : a.tokens;
  const int chunks = (int)((longest + MEM_CHUNK - 1) / MEM_CHUNK);
  const double room = 2. * cus / ((double)a.heads * slices);  // segments
  if (chunks <= 2 || a.sequences >= room) return chunks < 1 ? 1 : chunks;
  const double each = a.tokens == a.sequences * longest ? chunks / floor(room / a.sequences) : (double)a.tokens / MEM_CHUNK / (room - 0.5 * a.sequences);
  return (int)fmin(fmax(ceil(each), 2.), (double)chunks);
}

MemArgs forward_args(const ttc_linear_attention_t& a) {
  const int group = a.heads / a.heads_qk;
  MemArgs p = {};
  p.x = {a.q, a.q_token, a.q_head, group, a.dk};
  p.w = {a.k, a.k_token, a.k_head, group, a.dk};
  p.v = {a.v, a.v_token, a.v_head, 1, a.dv};
  p.out = a.out;
  p.out_token = a.out_token;
  p.out_head = a.out_head;
  p.heads = a.heads;
  p.pair_scale = p.in_scale = a.scale;
  p.up_scale = 1.f;
  p.log_decay = a.log_decay;
  p.g_token = a.g_token;
  p.g_head = a.g_head;
  p.states = {a.state_in, a.state_out, a.state_rows, a.state_row, a.kv_len};
  p.s_row = a.dv;
  p.s_col = 1;
  p.dk = a.dk;
  p.dv = a.dv;
  return p;
}

// One call, or two of the same sequences, heads and sizes
hipError_t run_chunks(const MemArgs& a, const MemArgs* b, bool bf16, int what, hipStream_t st) {
  const int rows = a.w.d, columns = columns_of(rows, a.v.d, bf16);
  MemTwo p = {{a, b ? *b : a}, 0};
  p.of[0].slices = p.of[1].slices = slices_of(rows, a.v.d, bf16);
  p.split = dealt(a.m, a.heads, p.of[0].slices);
  const uint32_t grid = b ? 2 * p.split : p.split;
  return rows <= 64 ? launch_memory_chunks<64>(p, bf16, columns, what, grid, st)
                    : rows <= 128 ? launch_memory_chunks<128>(p, bf16, columns, what, grid, st) : launch_memory_chunks<256>(p, bf16, columns, what, grid, st);
}

// What the segments add to their states, and from that what each finds
hipError_t run_starts(const MemArgs& a, const MemArgs* b, bool bf16, hipStream_t st) {
  if (const hipError_t e = run_chunks(a, b, bf16, MEM_STATES, st); e != hipSuccess) return e;
  const int64_t blocks = (a.dk * a.dv / 4 + 255) / 256;
  MemTwo p = {{a, b ? *b : a}, (uint32_t)(a.m.sequences * a.heads * blocks)};
  hipLaunchKernelGGL(memory_scan_kernel, dim3(b ? 2 * p.split : p.split), dim3(256), 0, st, p);
  return hipGetLastError();
}

uint64_t round16(uint64_t n) { return (n + 15) & ~15ull; }

}  // namespace

uint64_t linear_attention_workspace(const ttc_linear_attention_t& a, int cus) {
  if (a.max_q <= step_most(a.dtype == TTC_BF16)) return 0;
  const MemSequences m = sequences_of(a, segment_of(a, slices_of(a.dk, a.dv, a.dtype == TTC_BF16), cus), 1);
  if (m.entries == m.sequences) return 0;
  return (uint64_t)m.entries * a.heads * a.dk * a.dv * 4 + round16((uint64_t)m.entries * a.heads * 4);
}

hipError_t launch_linear_attention(const ttc_linear_attention_t& a, int cus, void* workspace, hipStream_t st) {
  const bool bf16 = a.dtype == TTC_BF16;
  MemArgs p = forward_args(a);
  if (a.max_q <= step_most(bf16)) {
    p.m = sequences_of(a, 1, 1);
    p.slices = (a.dv + 63) / 64;
    const uint32_t grid = (uint32_t)(a.sequences * a.heads * p.slices);
    return a.dk <= 64 ? launch_memory_step<64>(p, bf16, grid, st) : a.dk <= 128 ? launch_memory_step<128>(p, bf16, grid, st) : launch_memory_step<256>(p, bf16, grid, st);
  }
  p.m = sequences_of(a, segment_of(a, slices_of(a.dk, a.dv, a.dtype == TTC_BF16), cus), 1);
  if (p.m.entries != p.m.sequences) {
    p.added = static_cast<float*>(workspace);
    p.faded = p.added + p.m.entries * a.heads * a.dk * a.dv;
    if (const hipError_t e = run_starts(p, nullptr, bf16, st); e != hipSuccess) return e;
    p.starts = p.added;
  }
  return run_chunks(p, nullptr, bf16, MEM_OUT, st);
}

namespace {

// Places in the workspace of a backward pass, in bytes from its beginning
struct BackwardPlan {
  MemSequences m, chunks;
  int slices, pair_slices;  // of dq's and dk's columns, of dv's
  uint64_t added, faded, added_r, faded_r, a, b, pairs, gstate, sums, gq, gk, bytes;
};

BackwardPlan plan_backward(const ttc_linear_attention_backward_t& b, int cus) {
  const ttc_linear_attention_t& f = b.forward;
  BackwardPlan p = {};
  p.slices = slices_of(f.dv, f.dk, f.dtype == TTC_BF16);
  p.pair_slices = slices_of(f.dk, f.dv, f.dtype == TTC_BF16);
  p.m = sequences_of(f, segment_of(f, 2 * p.slices, cus), 1);  // (two calls are in a launch: 230 us for four times 2048 tokens; 245 with segments for one)
  p.chunks = sequences_of(f, 1, 8);
  uint64_t at = 0;
  const auto take = [&](uint64_t& place, uint64_t bytes) {
    place = at;
    at += round16(bytes);
  };
  const uint64_t state = (uint64_t)f.dk * f.dv * 4;
  if (p.m.entries != p.m.sequences) {
    take(p.added, p.m.entries * f.heads * state);
    take(p.faded, p.m.entries * f.heads * 4);
    take(p.added_r, p.m.entries * f.heads * state);
    take(p.faded_r, p.m.entries * f.heads * 4);
  }
  take(p.a, (uint64_t)p.slices * f.heads * f.tokens * 4);
  take(p.b, (uint64_t)p.slices * f.heads * f.tokens * 4);
  take(p.pairs, (uint64_t)p.pair_slices * f.heads * f.tokens * 4);
  if (f.state_in && !b.gstate) take(p.gstate, f.sequences * f.heads * state);
  if (!f.g_token) take(p.sums, (uint64_t)p.m.entries * f.heads * 8);
  if (f.heads != f.heads_qk) {
    take(p.gq, (uint64_t)f.tokens * f.heads * f.dk * 4);
    take(p.gk, (uint64_t)f.tokens * f.heads * f.dk * 4);
  }
  p.bytes = at;
  return p;
}

}  // namespace

uint64_t linear_attention_backward_workspace(const ttc_linear_attention_backward_t& b, int cus) { return plan_backward(b, cus).bytes; }

hipError_t launch_linear_attention_backward(const ttc_linear_attention_backward_t& b, int cus, void* workspace, hipStream_t st) {
  const ttc_linear_attention_t& f = b.forward;
  const BackwardPlan plan = plan_backward(b, cus);
  const bool bf16 = f.dtype == TTC_BF16, segmented = plan.m.entries != f.sequences;
  const int group = f.heads / f.heads_qk;
  char* const ws = static_cast<char*>(workspace);
  const auto place = [&](uint64_t at) { return reinterpret_cast<float*>(ws + at); };
  float* const gstate = b.gstate ? b.gstate : f.state_in ? place(plan.gstate) : nullptr;

  MemArgs base = forward_args(f);
  base.m = plan.m;
  base.states.out = nullptr;
  const MemRows q = base.x, k = base.w, v = base.v, gout = {b.gout, b.gout_token, b.gout_head, 1, f.dv};
  const MemStates begin = base.states, end = {b.gstate_out, gstate, f.sequences, nullptr, nullptr};
  MemArgs back = base;
  back.reverse = 1;
  back.states = end;
  back.rule = begin;
  back.ruled = 1;
  back.in_scale = 1.f;
  back.up_scale = f.scale;
  back.x = k;
  back.w = q;
  back.v = gout;
  hipError_t e;
  if (!f.sequences) {
    if (!f.g_token) hipLaunchKernelGGL(memory_decay_sum_kernel, dim3(f.heads), dim3(256), 0, st, nullptr, 0, f.heads, b.glog_decay);
    return hipGetLastError();
  }
  if (segmented) {
    base.added = place(plan.added);
    base.faded = place(plan.faded);
    back.added = place(plan.added_r);
    back.faded = place(plan.faded_r);
    if ((e = run_starts(base, &back, bf16, st)) != hipSuccess) return e;
    base.starts = base.added;
    back.starts = back.added;
  }
  const auto result = [&](MemArgs& p, void* out, uint64_t parts, int heads, int d) {
    const bool shared = heads != f.heads;
    p.out = shared ? ws + parts : out;
    p.out_float = shared;
    p.out_token = (int64_t)f.heads * d;
    p.out_head = d;
  };
  MemArgs dv = back;
  result(dv, b.gv, 0, f.heads, f.dv);
  dv.dot = v;
  dv.dots = place(plan.pairs);
  if ((e = run_chunks(dv, nullptr, bf16, MEM_OUT_PAIRS, st)) != hipSuccess) return e;
  MemArgs dk = back;
  dk.x = v;
  dk.w = gout;
  dk.v = q;
  dk.states.out = nullptr;
  dk.s_row = 1;
  dk.s_col = f.dv;
  dk.dot = k;
  dk.dots = place(plan.b);
  result(dk, b.gk, plan.gk, f.heads_qk, f.dk);
  MemArgs dq = base;
  dq.x = gout;
  dq.w = v;
  dq.v = k;
  dq.s_row = 1;
  dq.s_col = f.dv;
  dq.dot = q;
  dq.dots = place(plan.a);
  result(dq, b.gq, plan.gq, f.heads_qk, f.dk);
  if ((e = run_chunks(dk, &dq, bf16, MEM_OUT_DOTS, st)) != hipSuccess) return e;
  if (group > 1) {
    MemSequences m = plan.chunks;
    m.blocks = blocks_of(m.entries, f.heads_qk);
    const uint32_t split = dealt(m, f.heads_qk, 1);
    const auto run = [&](auto type) {
      typedef decltype(type) T;
      hipLaunchKernelGGL((memory_heads_kernel<T>), dim3(2 * split), dim3(256), 0, st, m, place(plan.gq), static_cast<T*>(b.gq), place(plan.gk),
                         static_cast<T*>(b.gk), split, f.heads_qk, group, f.dk);
    };
    if (bf16) run((unsigned short)0);
    else run(0.f);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  MemDecayArgs d = {};
  d.m = plan.m;
  d.heads = f.heads;
  d.dk = f.dk;
  d.dv = f.dv;
  d.slices = plan.slices;
  d.pair_slices = plan.pair_slices;
  d.pairs = place(plan.pairs);
  d.a = place(plan.a);
  d.b = place(plan.b);
  d.log_decay = f.log_decay;
  d.g_token = f.g_token;
  d.g_head = f.g_head;
  d.begin = begin;
  d.gstate = gstate;
  d.out = f.g_token ? b.glog_decay : nullptr;
  d.sums = f.g_token ? nullptr : reinterpret_cast<double*>(ws + plan.sums);
  d.found = base.starts;
  d.found_r = back.starts;
  hipLaunchKernelGGL(memory_decay_kernel, dim3((uint32_t)(plan.m.entries * f.heads)), dim3(MEM_SUM_THREADS), 0, st, d);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (!f.g_token) hipLaunchKernelGGL(memory_decay_sum_kernel, dim3(f.heads), dim3(256), 0, st, d.sums, plan.m.entries, f.heads, b.glog_decay);
  return hipGetLastError();
}

}  // namespace ttc
