// Attention over a paged cache: for query i of a sequence of n_q queries and L keys, over the keys j < lim_i,
//   x_j = scale q_i . k_j,  m = max x_j,  z = sum exp(x_j - m),  out = sum exp(x_j - m) v_j / z,  lse = m + log z,
// lim_i = L - n_q + i + 1 (causal: the queries are the sequence's last tokens) or L.  A row without keys gets out 0, lse -inf.
// Keys are taken once, in pieces: a piece's (m, z, unnormalised out) are joined by m = max m_p, z = sum z_p 2^(m_p - m) and the
// same for out (attend_plan.h: how the work is cut).  Logits are kept in units of log 2.
//
// Split items, for few rows: bound by reading K and V.  Each wavefront of the workgroup takes every fourth block of 32 keys (16 in fp32) of
// the item, for all rows of its tile, straight from memory into registers in the layout of the matrix instruction's operand:
//   x^T = K Q^T  (v_mfma_f32_16x16x32_bf16; lane (r = lane % 16, g = lane / 16) holds K[r][8 g ..]),
//   out^T += V^T P^T.
// The accumulator has the query in lane % 16 and keys 4 g .. 4 g + 3, so softmax statistics stay within a lane, and the
// probabilities are the second product's operand where they stand, if the contraction takes the keys in the order
// slot (g, j) = key 16 (j / 4) + 4 g + j % 4.  V rows are loaded in that order, 16 bytes of a row a lane, and turned with byte
// permutes in registers: no LDS and no barrier until the four wavefronts join their results.  One token over 131089 keys, 28 and 4
// heads of 128: 268 MB in 47 us = 5.7 TB/s.
//
// Tile items, for many rows (bf16, d <= 128): bound by the products.  Each wavefront has 16 MT rows of its own, and all four take the
// same tiles of 64 keys from LDS, which are loaded there directly, into one of two buffers while the other is worked on: K as it
// stands as an operand (lane by lane), V by rows with their 16-byte pieces exchanged, so that the transposing reads that
// make operands of it (ds_read_b64_tr_b16) have no bank conflicts either.  A chunk of 3565 tokens over 14 to 16 thousand keys, 32 and
// 8 heads of 128: 862 us = 857 TFLOP/s of the keys that are seen (a library product of 8192^3: 1210); products, exponentials and
// LDS reads, each about a third of the cycles, overlap only between the two workgroups of a unit.
#pragma once
#include "paged.h"

#include "asl_internal.h"
#include "attend_plan.h"

namespace asl {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t Piece __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// A row's reference moves when a logit exceeds it by more than this (in units of log 2): probabilities stay below 2^8 and most
// blocks need no maximum over lanes and no rescaling.
constexpr float kSlack = 8.f;
// The same where a row's reference cannot move in place: probabilities up to 2^24 lose nothing in fp32 and bf16 (a result is a
// quotient of two such sums; over n keys sums of values below 2^103 / n stay below 2^128), and only rows whose first tile was that
// much lower than a later one need the step that moves it.
constexpr float kWideSlack = 24.f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void paged_fault(const PageMap& m) { atomicOr(m.fault, kFaultPaged); }

// Maximum / sum over the four lanes that share lane % 16.
__device__ __forceinline__ float max_over_g(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_g(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// sequence_of by a whole wavefront: a load for up to 64 sequences, two for up to 4096, where a binary search waits for one after another.
__device__ __forceinline__ int sequence_by_wave(const int32_t* cu, int n, int j) {
  const int lane = threadIdx.x & 63, step = (n + 63) / 64;
  int first = 0;
  if (step > 1) {
    const int i = lane * step;
    first = step * max(0, (int)__popcll(__ballot(i < n && cu[min(i, n - 1)] <= j)) - 1);
  }
  const int i = first + lane;
  return min(n - 1, first + max(0, (int)__popcll(__ballot(i < n && lane < step + (step == 1 ? 63 : 0) && cu[min(i, n - 1)] <= j)) - 1));
}

// ------------------------------------------------------------------------------------------------------------------
// The cut, found by every wavefront for itself.

struct Segment {
  int c0, rows;            // first query token, rows of a KV head
  int row, len;            // table row and its tokens
  int t0, span;            // first key tile and number of key tiles
  int shared;              // own segments: tokens in the group's shared segment
  int b0, b1;              // shared segments: the group's sequences
  int group;               // own segments: the sequence's, or -1
};

__device__ __forceinline__ int seq_row(const AttendArgs& a, int b) { return a.rows != nullptr ? a.rows[b] : b; }

// Tokens shared by group g.
__device__ __forceinline__ int group_shared(const AttendArgs& a, int g) {
  const int b0 = a.group_start[g], b1 = a.group_start[g + 1];
  if (b0 < 0 || b1 <= b0 || b1 > a.n_seqs) return 0;
  int len;
  row_length(a.map, seq_row(a, b0), &len);
  return shared_tokens(a.prefix_len[g], len, b1 - b0);
}

// Up to 64 groups, a lane each: an own segment finds its group and the shared tokens among the lanes, where loads would wait for one
// another (search, group, first sequence, its length).
struct Groups {
  int start, end, shared;
  bool in_lanes, on;       // on: the groups together save enough

  __device__ __forceinline__ Groups(const AttendArgs& a) {
    const int lane = threadIdx.x & 63;
    start = end = shared = 0;
    in_lanes = a.n_groups <= 64;
    on = false;
    if (a.n_groups == 0) return;
    unsigned long long saved = 0;                          // keys
    for (int g = lane; g < a.n_groups; g += 64) {
      start = a.group_start[g];
      end = a.group_start[g + 1];
      shared = group_shared(a, g);
      saved += (unsigned long long)max(0, end - start - 1) * (uint32_t)shared;
    }
    on = groups_pay(wave_sum(saved), a.key_bytes);
  }
  // The group of sequence b, or -1; *tokens: what it shares.  (Every lane of the wavefront calls it.)
  __device__ __forceinline__ int find(const AttendArgs& a, int b, int* tokens) const {
    int g, first, last;
    if (in_lanes) {
      g = 0;
      for (int k = 1; k < a.n_groups; ++k) g = __builtin_amdgcn_readlane(start, k) <= b ? k : g;
      first = __shfl(start, g);
      last = __shfl(end, g);
      *tokens = __shfl(shared, g);
    } else {
      b = min(max(b, 0), a.n_seqs - 1);
      g = sequence_of(a.group_start, a.n_groups, b);
      first = a.group_start[g];
      last = a.group_start[g + 1];
      *tokens = group_shared(a, g);
    }
    if (first <= b && b < last) return g;
    *tokens = 0;
    return -1;
  }
};

// Segment i: sequence i's own (SHARED false), or group i's shared one.  *bad: a number out of range.
// (Every lane of the wavefront calls it; those with i out of range get an empty one.)
template <bool SHARED>
__device__ __forceinline__ Segment segment_of(const AttendArgs& a, const Groups& groups, int i, bool* bad) {
  Segment s = {};
  s.group = -1;
  int tokens = 0;
  if (!SHARED && a.n_groups > 0) s.group = groups.find(a, i, &tokens);
  if (!groups.on) tokens = 0;
  if (SHARED && !groups.on) return s;
  if (i >= (SHARED ? a.n_groups : a.n_seqs)) return s;
  if (SHARED) {
    const int p = group_shared(a, i);
    if (p == 0) return s;
    const int b0 = a.group_start[i], b1 = a.group_start[i + 1], c0 = a.cu_q[b0], c1 = a.cu_q[b1];
    if (c0 < 0 || c1 < c0 || c1 > a.total_q) { *bad = true; return s; }
    s.c0 = c0;
    s.rows = (c1 - c0) * a.G;
    s.row = seq_row(a, b0);
    s.len = p;
    s.span = p / kKeyTile;
    s.b0 = b0;
    s.b1 = b1;
    return s;
  }
  const int c0 = a.cu_q[i], c1 = a.cu_q[i + 1];
  s.row = seq_row(a, i);
  if (!row_length(a.map, s.row, &s.len)) *bad = true;
  if (c0 < 0 || c1 < c0 || c1 > a.total_q) { *bad = true; return s; }
  s.c0 = c0;
  s.rows = (c1 - c0) * a.G;
  if (a.n_groups > 0) {
    if (s.group < 0) *bad = true;
    s.shared = tokens;
  }
  s.t0 = s.shared / kKeyTile;
  s.span = max(0, (s.len + kKeyTile - 1) / kKeyTile - s.t0);
  return s;
}

struct Partials {
  float* o;                // [cap][D]
  float2* mz;              // [cap]
  int4* plan;              // of the segments
  int32_t* group;          // [n_seqs] own segments: the sequence's group or -1
  int32_t* cut;            // own segments: whether any row is in pieces
  uint32_t* arrived;       // [cap] zeros: pieces of a row tile that are there, counted at its first slot; null: a launch joins them
};

struct Item {
  Segment seg;
  int tile, h, split, splits;
  int64_t slot;            // of the segment's first row of partial results, or -1: the results are whole
};

// What the joining kernel has to know of a segment: first token, rows, splits (0: nothing to join) and first slot.
__device__ __forceinline__ int4 plan_entry(const Segment& s, int splits, bool partial, uint32_t slot) {
  return make_int4(s.c0, s.rows, partial ? splits : 0, (int)slot);
}

template <bool SHARED>
__device__ __forceinline__ bool find_item(const AttendArgs& a, const AttendCut& cut, int item, const Partials& pt, Item* out) {
  const int lane = threadIdx.x & 63;
  const int n = SHARED ? a.n_groups : a.n_seqs, per = (n + 63) / 64;
  const bool writes = item == 0 && threadIdx.x < 64;
  bool bad = false;
  auto row_tiles = [&](const Segment& s) { return (uint32_t)((s.rows + cut.rows - 1) / cut.rows) * (uint32_t)a.Hk; };
  auto is_partial = [&](const Segment& s, int splits) { return SHARED || splits > 1 || s.shared > 0; };
  Segment own = {};
  const Groups groups(a);
  unsigned long long work = 0, all_rows = 0;
  for (int u = 0; u < per; ++u) {
    own = segment_of<SHARED>(a, groups, lane * per + u, &bad);
    all_rows += (unsigned long long)own.rows;
    work += (unsigned long long)row_tiles(own) * (uint32_t)max(own.span, 1);   // (no rows: 0)
  }
  // Lists that do not ascend can have a token in several sequences: more rows than the launch, the pieces' room and their counts are
  // made for.  Nothing is done then.
  const bool sound = wave_sum(all_rows) <= (unsigned long long)a.total_q * (unsigned long long)a.G;
  if (writes && (bad || !sound)) paged_fault(a.map);
  if (!sound) {
    if (writes) {
      for (int i = lane; i < n; i += 64) pt.plan[i] = make_int4(0, 0, 0, 0);
      if (!SHARED && lane == 0) *pt.cut = 0;
    }
    return false;
  }
  int64_t per_item = tiles_per_item(cut, wave_sum(work));
  uint32_t items, slots, upto, slots_upto;
  for (int round = 0;; ++round) {
    items = slots = 0;
    for (int u = 0; u < per; ++u) {
      if (per > 1) own = segment_of<SHARED>(a, groups, lane * per + u, &bad);
      const int k = splits_of(own.span, per_item);
      items += row_tiles(own) * (uint32_t)k;
      slots += is_partial(own, k) ? (uint32_t)own.rows * (uint32_t)a.Hk * (uint32_t)k : 0u;
    }
    upto = wave_prefix_sum(items);
    slots_upto = wave_prefix_sum(slots);
    if (round > 0 || (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)slots_upto, 63) <= cut.cap) break;
    per_item = int64_t(1) << 40;                           // no room for the pieces: whole spans
  }
  if (writes) {
    if (!SHARED && lane == 63) *pt.cut = slots_upto != 0 ? 1 : 0;
    uint32_t at = slots_upto - slots;
    for (int u = 0; u < per; ++u) {
      const int i = lane * per + u;
      if (per > 1) own = segment_of<SHARED>(a, groups, i, &bad);
      if (i >= n) continue;
      const int k = splits_of(own.span, per_item);
      const bool partial = is_partial(own, k);
      pt.plan[i] = plan_entry(own, k, partial && own.rows > 0, at);
      if (!SHARED && a.n_groups > 0) pt.group[i] = own.group;
      if (partial) at += (uint32_t)own.rows * (uint32_t)a.Hk * (uint32_t)k;
    }
  }
  const uint64_t past = __ballot(upto > (uint32_t)item);
  if (past == 0) return false;
  const int l = __ffsll((unsigned long long)past) - 1;
  uint32_t base = (uint32_t)__builtin_amdgcn_readlane((int)(upto - items), l);
  uint32_t slot = (uint32_t)__builtin_amdgcn_readlane((int)(slots_upto - slots), l);
  int from = l;
  if (per > 1) {                                           // the same among the lane's segments (per <= 64)
    const int i = l * per + lane;
    items = slots = 0;
    own = segment_of<SHARED>(a, groups, lane < per ? i : n, &bad);
    if (lane < per && i < n) {
      const int k = splits_of(own.span, per_item);
      items = row_tiles(own) * (uint32_t)k;
      slots = is_partial(own, k) ? (uint32_t)own.rows * (uint32_t)a.Hk * (uint32_t)k : 0u;
    }
    upto = wave_prefix_sum(items);
    slots_upto = wave_prefix_sum(slots);
    const uint64_t more = __ballot(base + upto > (uint32_t)item);
    if (more == 0) return false;
    from = __ffsll((unsigned long long)more) - 1;
    base += (uint32_t)__builtin_amdgcn_readlane((int)(upto - items), from);
    slot += (uint32_t)__builtin_amdgcn_readlane((int)(slots_upto - slots), from);
  }
  Segment s;
  s.c0 = __builtin_amdgcn_readlane(own.c0, from);
  s.rows = __builtin_amdgcn_readlane(own.rows, from);
  s.row = __builtin_amdgcn_readlane(own.row, from);
  s.len = __builtin_amdgcn_readlane(own.len, from);
  s.t0 = __builtin_amdgcn_readlane(own.t0, from);
  s.span = __builtin_amdgcn_readlane(own.span, from);
  s.shared = __builtin_amdgcn_readlane(own.shared, from);
  s.b0 = __builtin_amdgcn_readlane(own.b0, from);
  s.b1 = __builtin_amdgcn_readlane(own.b1, from);
  out->seg = s;
  out->splits = splits_of(s.span, per_item);
  const uint32_t e = (uint32_t)item - base, tiles = (uint32_t)((s.rows + cut.rows - 1) / cut.rows);
  out->h = (int)(e % (uint32_t)a.Hk);
  out->tile = (int)(tiles - 1u - (e / (uint32_t)a.Hk) % tiles);    // causal: the longest first
  out->split = (int)(e / (uint32_t)a.Hk / tiles);
  out->slot = is_partial(s, out->splits) ? (int64_t)slot : -1;
  return out->slot < 0 || (int64_t)slot + (int64_t)s.rows * a.Hk * out->splits <= cut.cap;
}

// The fewest keys that a row of a shared segment's sequences sees, or the segment's if that is less: found by lanes over the sequences,
// since a row's own takes a search for its sequence.
__device__ __forceinline__ int least_limit(const AttendArgs& a, const Segment& s) {
  uint32_t least = (uint32_t)s.len;
  for (int b = s.b0 + (int)(threadIdx.x & 63); b < s.b1; b += 64) {
    const int n = a.cu_q[b + 1] - a.cu_q[b];
    int len;
    row_length(a.map, seq_row(a, b), &len);
    if (n > 0) least = min(least, (uint32_t)(a.causal ? max(0, len - n + 1) : len));
  }
  return (int)wave_min(least);
}

// Keys that row r of a segment sees.  all: as many as every row of a shared segment sees.
template <bool SHARED>
__device__ __forceinline__ int row_limit(const AttendArgs& a, const Segment& s, int r, int all) {
  const int i = (int)((uint32_t)r / (uint32_t)a.G);
  if (!SHARED) return a.causal ? max(0, s.len - s.rows / a.G + i + 1) : s.len;
  if (all == s.len) return s.len;
  const int tok = s.c0 + i, b = sequence_of(a.cu_q, a.n_seqs, tok);
  int len;
  row_length(a.map, seq_row(a, b), &len);
  return min(s.len, a.causal ? max(0, len - (a.cu_q[b + 1] - tok) + 1) : len);
}

// ------------------------------------------------------------------------------------------------------------------
// Registers of a block of keys, and the arithmetic on them.

template <typename T, int D>
struct Block {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int SUB = kBf16 ? 2 : 1;                // subtiles of 16 keys
  static constexpr int KEYS = 16 * SUB;
  static constexpr int KP = D * (int)sizeof(T) / 64;       // 16-byte pieces of K a lane holds of a subtile
  static constexpr int VR = KEYS / 4;                      // rows of V that a lane holds parts of
  static constexpr int CW = kBf16 && D >= 128 ? 8 : 4;     // consecutive elements of each
  static constexpr int VW = CW * (int)sizeof(T) / 4;       // in words
  static constexpr int HN = D / (16 * CW);                 // parts of a row: element 16 CW hf + CW (lane % 16) + e
  static constexpr int NT = D / 16;                        // accumulators of out: index hf * CW + e
  Piece k[SUB][KP];
  uint32_t v[VR][HN][VW];
  bool ok[SUB];                                            // the subtile's page number is in range

  // Key of row j of V within the block.
  static __device__ __forceinline__ int v_key(int j, int g) { return 16 * (j >> 2) + 4 * g + (j & 3); }
};

struct Source {
  const char* k;           // pages of the KV head
  const char* v;
  const int32_t* table;    // the segment's row
  int64_t page, tok;
  int n_pages, ps, shift, last;    // last: the last key's subtile (no page number behind it is read)
  int d;
};

// A uniform address, kept in scalar registers: lanes add 32-bit offsets to it.  (Without this the compiler adds the lanes' offsets to the
// pages' address ahead of the loop, and keeps 64-bit sums in vector registers.)
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t x = (uint64_t)p;
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32));
  return (const char*)(((uint64_t)hi << 32) | lo);
}

// A lane's 32-bit offset where it is used: the compiler would widen it ahead of the loop, and then add 64 bits.
__device__ __forceinline__ uint32_t offset(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Elements e0 .. e0 + CW - 1 of the row at base + row, zeros beyond d.
template <typename T, int D, bool PAD, bool STREAM>
__device__ __forceinline__ void load_value(uint32_t* to, const char* base, uint32_t row, int e0, int d) {
  typedef uint32_t Words __attribute__((ext_vector_type(Block<T, D>::VW)));
  const bool in = !PAD || e0 < d;
  const Words* from = (const Words*)(base + (row + (uint32_t)(in ? e0 : 0) * (uint32_t)sizeof(T)));
  const Words w = STREAM ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
  for (int x = 0; x < Block<T, D>::VW; ++x) to[x] = in ? w[x] : 0u;
}

// Page numbers of the blocks that a wavefront comes to, each STEP keys behind the last and of SUB subtiles: 64 of them at a time, a lane
// each, and the 64 behind them already on their way.  (A load for each block would be waited for before the block's own
// loads can go out: the prefill chunk took 3239 us with it when it took 2680 without.)
template <int SUB, int STEP>
struct PageWindow {
  static constexpr int kBlocks = 64 / SUB;
  int cur, nxt, key, first;    // key: of block 0; first: block of cur's first lane

  __device__ __forceinline__ int fetch(const Source& s, int block) const {
    const int lane = threadIdx.x & 63;
    const int k = min(key + (block + lane / SUB) * STEP + 16 * (lane % SUB), s.last);
    return s.table[k >> s.shift];
  }
  __device__ __forceinline__ void start(const Source& s, int key0) {
    key = key0;
    first = 0;
    cur = fetch(s, 0);
    nxt = fetch(s, kBlocks);
  }
  __device__ __forceinline__ void move(const Source& s, int block) {
    if (block - first < kBlocks) return;
    cur = nxt;
    first += kBlocks;
    nxt = fetch(s, first + kBlocks);
  }
  __device__ __forceinline__ int page(int block, int t) const {
    const int l = (block - first) * SUB + t;
    const int from = l < 64 ? cur : nxt;
    return __builtin_amdgcn_readlane(from, l & 63);
  }
};

// STREAM: past the caches, for keys that one tile of rows takes (decode of 128K keys 58.7 us, so 53.2; a pruned batch 95.9, 87.8).
template <typename T, int D, bool PAD, bool STREAM, typename W>
__device__ __forceinline__ void load_block(Block<T, D>& b, const Source& s, const W& window, int block, int key0) {
  typedef Block<T, D> B;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const char* base[B::SUB];
#pragma unroll
  for (int t = 0; t < B::SUB; ++t) {
    const int key = min(key0 + 16 * t, s.last);
    const int page = window.page(block, t);
    b.ok[t] = (uint32_t)page < (uint32_t)s.n_pages;
    const int64_t off = (int64_t)(b.ok[t] ? page : 0) * s.page + (int64_t)(key & (s.ps - 1)) * s.tok;
    base[t] = uniform(s.v + off);
    const char* kb = uniform(s.k + off);
    const uint32_t ko = (uint32_t)r * (uint32_t)s.tok + (uint32_t)g * 16u;
#pragma unroll
    for (int p = 0; p < B::KP; ++p) {
      const bool in = !PAD || p * 64 + g * 16 < s.d * (int)sizeof(T);    // beyond d: the row's first piece, then zeros
      const Piece* from = (const Piece*)(kb + (in ? ko + p * 64u : (uint32_t)r * (uint32_t)s.tok));
      const Piece x = STREAM ? __builtin_nontemporal_load(from) : *from;
      b.k[t][p] = in ? x : Piece{0, 0, 0, 0};
    }
  }
#pragma unroll
  for (int j = 0; j < B::VR; ++j) {
#pragma unroll
    for (int hf = 0; hf < B::HN; ++hf)
      load_value<T, D, PAD, STREAM>(b.v[j][hf], base[j >> 2], (uint32_t)(4 * g + (j & 3)) * (uint32_t)s.tok, 16 * B::CW * hf + B::CW * r, s.d);
  }
}

// The sign bit of each element of a word that is infinite or NaN (its exponent, all ones, carries into the sign's place).
template <typename T> __device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return sizeof(T) == 2 ? ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u : ((w & 0x7f800000u) + 0x00800000u) & 0x80000000u;
}
// All bits of the elements whose sign bit is set in `bits`.
template <typename T> __device__ __forceinline__ uint32_t whole_elements(uint32_t bits) {
  return sizeof(T) == 2 ? (bits - (bits >> 15)) | bits : (bits - (bits >> 31)) | bits;
}
// One for each element of a word that is of class c (0: +inf, 1: -inf, 2: NaN), else zero.
template <typename T> __device__ __forceinline__ uint32_t word_class(uint32_t w, int c) {
  const uint32_t sign = sizeof(T) == 2 ? 0x80008000u : 0x80000000u, top = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u;
  const uint32_t frac = ~(sign | top), one = sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u;
  const uint32_t odd = whole_elements<T>(not_finite<T>(w));
  // a carry out of the fraction: it is not zero
  const uint32_t is_nan = whole_elements<T>((((w & frac) + frac) & (sizeof(T) == 2 ? 0x00800080u : 0x00800000u)) << 8);
  const uint32_t neg = whole_elements<T>(w & sign);
  const uint32_t is = c == 2 ? is_nan : c == 1 ? neg & ~is_nan : ~neg & ~is_nan;
  return odd & is & one;
}

// Element e of eight rows' words as an operand: rows 2 p and 2 p + 1 in word p.
__device__ __forceinline__ bf16x8 turn(const uint32_t (&w)[8], int odd) {
  const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
  union { uint32_t u[4]; bf16x8 v; } x;
#pragma unroll
  for (int p = 0; p < 4; ++p) x.u[p] = __builtin_amdgcn_perm(w[2 * p + 1], w[2 * p], sel);
  return x.v;
}

// Probabilities as the second product's operand.  (bf16: each rounds to 8 bits, so out is off by at most 2^-8 sum p |v| / z; a split in
// two parts would take twice the products.  The sum z is that of the unrounded ones.)
template <typename T> struct Weights;
template <> struct Weights<__bf16> {
  bf16x8 w;
  __device__ __forceinline__ void set(const float (&p)[2][4]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (__bf16)p[j >> 2][j & 3];
  }
};
template <> struct Weights<float> {
  float w[4];
  __device__ __forceinline__ void set(const float (&p)[1][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = p[0][i];
  }
};

// out[mt] + V^T p for part hf, element e of the rows of V, whose words are word(j, hf, x).
template <typename T, int MT, typename W>
__device__ __forceinline__ void add_values(f32x4* (&o)[MT], const Weights<T> (&p)[MT], int hf, int e, W word) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[8] = {word(0, hf, e / 2), word(1, hf, e / 2), word(2, hf, e / 2), word(3, hf, e / 2),
                           word(4, hf, e / 2), word(5, hf, e / 2), word(6, hf, e / 2), word(7, hf, e / 2)};
    const bf16x8 va = turn(w, e & 1);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p[mt].w, *o[mt], 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        *o[mt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(i, hf, e)), p[mt].w[i], *o[mt], 0, 0, 0);
  }
}

// A wavefront's running results for MT tiles of 16 rows.
template <typename T, int D, int MT>
struct Rows {
  typedef Block<T, D> B;
  Piece q[MT][B::KP];
  f32x4 o[MT][B::NT];
  float m[MT], z[MT];      // reference and, of this lane's keys, sum
  int lim[MT];
  uint32_t odd;            // values were left out

  __device__ __forceinline__ void clear() {
    odd = 0;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt] = -INFINITY;
      z[mt] = 0.f;
#pragma unroll
      for (int t = 0; t < B::NT; ++t) o[mt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // MASKED: some row does not see some key of the block.  most: keys that any row sees.
  template <bool MASKED>
  __device__ __forceinline__ void step(Block<T, D>& b, int key0, int least, int most, float scale) {
    const int g = (threadIdx.x & 63) >> 4;
    f32x4 x[MT][B::SUB];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int t = 0; t < B::SUB; ++t) x[mt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (B::kBf16) {
#pragma unroll
      for (int p = 0; p < B::KP; ++p)
#pragma unroll
        for (int t = 0; t < B::SUB; ++t)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b.k[t][p]),
                                                               __builtin_bit_cast(bf16x8, q[mt][p]), x[mt][t], 0, 0, 0);
    } else {
      // A score is summed in four chains of d / 16 instructions, since a chain's roundings grow with its length and a score's error is its
      // probability's.  Relative error of out against 64 bits at 300 .. 20000 keys, one chain / four: 4.8e-7 .. 8.9e-7 / 2.6e-7 .. 5.1e-7
      // for d = 64, 1.0e-6 .. 1.6e-6 / 3.7e-7 .. 6.4e-7 for d = 256.  One chain after the other, over neighbouring elements: with all
      // four open the kernels of d = 128 spill (3 x 100 rows of 16 heads on 3000 keys 149 us, so 141, one chain 143; 16 sequences of 3000
      // keys 45.6, 43.5, 44.1).  (Summing out by blocks of 16 keys as well takes 5.6e-7 to 4.6e-7 there, but half as long again.)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < B::SUB; ++t) {
          f32x4 pair = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = c * B::KP / 4; p < (c + 1) * B::KP / 4; ++p)
#pragma unroll
              for (int u = 0; u < 4; ++u)
                y = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.k[t][p][u]), __uint_as_float(q[mt][p][u]), y, 0, 0, 0);
            pair = c % 2 == 0 ? y : pair + y;
            if (c == 1) x[mt][t] = pair;
          }
          x[mt][t] += pair;
        }
    }
    float p[MT][B::SUB][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < B::SUB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = x[mt][t][i] * scale;
          if (MASKED) y = b.ok[t] && key0 + 16 * t + 4 * g + i < lim[mt] ? y : -INFINITY;
          p[mt][t][i] = y;
          top = fmaxf(top, y);
        }
      if (__any(top > m[mt] + kSlack)) {
        const float to = fmaxf(m[mt], max_over_g(top));
        const float by = to == -INFINITY ? 1.f : exp2_fast(m[mt] - to);
        m[mt] = to;
        z[mt] *= by;
#pragma unroll
        for (int t = 0; t < B::NT; ++t) o[mt][t] *= by;
      }
      const float base = m[mt] == -INFINITY ? 0.f : m[mt];
#pragma unroll
      for (int t = 0; t < B::SUB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[mt][t][i] = exp2_fast(p[mt][t][i] - base);
          z[mt] += p[mt][t][i];
        }
    }
    Weights<T> w[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) w[mt].set(p[mt]);
    add<MASKED>(b.v, b.ok[0], b.ok[B::SUB - 1], key0, least, most, w);
  }

  // out += V^T w for a block of values, whose subtiles' page numbers are in range or not (ok0, ok1).
  template <bool MASKED>
  __device__ __forceinline__ void add(uint32_t (&v)[B::VR][B::HN][B::VW], bool ok0, bool ok1, int key0, int least, int most,
                                      const Weights<T> (&w)[MT]) {
    const int g = (threadIdx.x & 63) >> 4;
    if (MASKED) {
      // Probability 0 does not keep a value that is no number out of the sum.  Behind the last key that any row sees, and in pages out
      // of range, values are replaced by zero; where rows differ in what they see, infinities and NaN are too, and add_odd
      // brings them back for the rows that see them.
      const bool differ = least < most;
#pragma unroll
      for (int j = 0; j < B::VR; ++j) {
        const uint32_t seen = ((j >> 2) == 0 ? ok0 : ok1) && key0 + B::v_key(j, g) < most ? ~0u : 0u;
#pragma unroll
        for (int hf = 0; hf < B::HN; ++hf)
#pragma unroll
          for (int x2 = 0; x2 < B::VW; ++x2) {
            uint32_t y = v[j][hf][x2] & seen;
            if (differ) {
              const uint32_t bits = not_finite<T>(y);
              odd |= bits;
              y &= ~whole_elements<T>(bits);
            }
            v[j][hf][x2] = y;
          }
      }
    }
#pragma unroll
    for (int hf = 0; hf < B::HN; ++hf)
#pragma unroll
      for (int e = 0; e < B::CW; ++e) {
        f32x4* to[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) to[mt] = &o[mt][hf * B::CW + e];
        add_values<T, MT>(to, w, hf, e, [&](int j, int hf2, int x2) { return v[j][hf2][x2]; });
      }
  }

  // Infinite values and NaN of the blocks at key0, key0 + step, ... before end, which the masked steps left out: counted by class for the
  // rows that see them, as a product of zeros and ones, and each class added as itself.  (Rare, and apart from the steps:
  // within them it would take their registers.)  ROWWISE: accumulator t has elements 16 t .. 16 t + 15 of out.
  template <bool ROWWISE>
  __device__ __forceinline__ void add_odd(const Source& s, int key0, int step, int end, int most) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll 1
    for (; key0 < end; key0 += step) {
      bool ok[B::SUB];
      const char* base[B::SUB];
      Weights<T> see[MT];
#pragma unroll
      for (int t = 0; t < B::SUB; ++t) {
        const int key = min(key0 + 16 * t, s.last);
        const int page = __builtin_amdgcn_readfirstlane(s.table[key >> s.shift]);
        ok[t] = (uint32_t)page < (uint32_t)s.n_pages;
        base[t] = s.v + (int64_t)(ok[t] ? page : 0) * s.page + (int64_t)(key & (s.ps - 1)) * s.tok;
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float one[B::SUB][4];
#pragma unroll
        for (int t = 0; t < B::SUB; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) one[t][i] = ok[t] && key0 + 16 * t + 4 * g + i < lim[mt] ? 1.f : 0.f;
        see[mt].set(one);
      }
#pragma unroll
      for (int t = 0; t < B::NT; ++t) {
        const int e = ROWWISE ? 16 * t + r : 16 * B::CW * (t / B::CW) + B::CW * r + t % B::CW;
        uint32_t v[B::VR], any = 0;                        // the element of each key's row, alone in a word
#pragma unroll
        for (int j = 0; j < B::VR; ++j) {
          v[j] = 0;
          if (ok[j >> 2] && key0 + B::v_key(j, g) < most && e < s.d) {
            const char* at = base[j >> 2] + (int64_t)(4 * g + (j & 3)) * s.tok + (int64_t)e * (int)sizeof(T);
            v[j] = B::kBf16 ? (uint32_t)*(const uint16_t*)at : *(const uint32_t*)at;
          }
          any |= not_finite<T>(v[j]);
        }
        if (!__any(any != 0)) continue;
#pragma unroll 1
        for (int c = 0; c < 3; ++c) {
          const float what = c == 0 ? INFINITY : c == 1 ? -INFINITY : __uint_as_float(0x7fc00000u);
          f32x4 n[MT];
          f32x4* to[MT];
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            n[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
            to[mt] = &n[mt];
          }
          // (turn(): the even element of each word)
          add_values<T, MT>(to, see, 0, 0, [&](int j, int, int) { return word_class<T>(v[j], c); });
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[mt][t][i] += n[mt][i] > 0.f ? what : 0.f;
        }
      }
    }
  }
};

// ------------------------------------------------------------------------------------------------------------------


// Two floats written through, and read past, this die's caches (device-scope atomic accesses).
__device__ __forceinline__ void store_through(float* p, float x, float y) {
  const unsigned long long w = ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x);
  __hip_atomic_store((unsigned long long*)p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_through(const float* p) {
  const unsigned long long w = __hip_atomic_load((const unsigned long long*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
}

// Writes row r of an item: to out and lse if its results are whole, else to its slot.  v: CNT elements from e0 on.
template <typename T, int CNT>
__device__ __forceinline__ void write_row(const AttendArgs& a, const Item& it, const Partials& pt, int D, int r, int e0,
                                          const float (&v)[CNT], float m, float z) {
  if (it.slot >= 0) {
    const int64_t slot = it.slot + ((int64_t)it.h * it.splits + it.split) * it.seg.rows + r;
    if (pt.arrived != nullptr) {                           // for another workgroup of this launch: see join_last
#pragma unroll
      for (int x = 0; x < CNT; x += 2) store_through(pt.o + slot * D + e0 + x, v[x], v[x + 1]);
      if (e0 == 0) store_through((float*)(pt.mz + slot), m, z);
      return;
    }
#pragma unroll
    for (int x = 0; x < CNT; x += 4) *(f32x4*)(pt.o + slot * D + e0 + x) = f32x4{v[x], v[x + 1], v[x + 2], v[x + 3]};
    if (e0 == 0) pt.mz[slot] = make_float2(m, z);
    return;
  }
  const int i = (int)((uint32_t)r / (uint32_t)a.G), tok = it.seg.c0 + i, hq = it.h * a.G + (r - i * a.G);
  const float by = z == 0.f ? 0.f : 1.f / z;               // no key: the sums are zero
  T* to = (T*)a.out + (int64_t)tok * a.ot + (int64_t)hq * a.oh + e0;
  constexpr int W = store_elements(CNT, (int)sizeof(T));
  typedef T Out __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int x0 = 0; x0 < CNT; x0 += W) {
    Out w;
#pragma unroll
    for (int x = 0; x < W; ++x) w[x] = (T)(v[x0 + x] * by);
    if (e0 + x0 < a.d) *(Out*)(to + x0) = w;
  }
  if (e0 == 0 && a.lse != nullptr) a.lse[(int64_t)hq * a.total_q + tok] = z == 0.f ? -INFINITY : (m + __log2f(z)) * kLn2;
}

__device__ __forceinline__ Source source_of(const AttendArgs& a, const Item& it) {
  Source src;
  src.k = (const char*)a.k + (int64_t)it.h * a.map.head;
  src.v = (const char*)a.v + (int64_t)it.h * a.map.head;
  src.table = a.map.table + (int64_t)it.seg.row * a.map.row_stride;
  src.page = a.map.page;
  src.tok = a.map.tok;
  src.n_pages = a.map.n_pages;
  src.ps = a.map.ps;
  src.shift = a.map.ps_shift;
  src.last = (it.seg.len - 1) & ~15;
  src.d = a.d;
  return src;
}

// Key tiles [*t0, *t1) of an item: its share of those that any of its rows sees (of a shared segment: of all).
template <bool SHARED>
__device__ __forceinline__ void tiles_of(const AttendArgs& a, const Item& it, int tile_rows, int* t0, int* t1) {
  int any = it.seg.len;
  if (!SHARED) any = row_limit<false>(a, it.seg, min(it.seg.rows, (it.tile + 1) * tile_rows) - 1, 0);
  split_range(min(it.seg.span, max(0, (any + kKeyTile - 1) / kKeyTile - it.seg.t0)), it.splits, it.split, t0, t1);
  *t0 += it.seg.t0;
  *t1 += it.seg.t0;
}

// The workgroup that brings the last piece of a tile of 16 rows joins them, 16 threads a row (few pieces: the launch that joins many
// would take longer to begin than this takes).  Pieces are written through to memory, every wavefront waits until its own are
// there, then one thread counts the workgroup's in; whoever counts the last one reads them past its caches.  (With
// fences instead, which write a die's whole cache back, 8 sequences of 1024 keys took 40 us instead of 13.)  The
// count is put back to 0 for the next call.
template <typename T, int D>
__device__ __forceinline__ void join_last(const AttendArgs& a, const AttendCut& cut, const Partials& pt, const Item& it, uint32_t* lds) {
  const int64_t first = it.slot + (int64_t)it.h * it.splits * it.seg.rows + it.tile * cut.rows;
  __builtin_amdgcn_s_waitcnt(0);                           // this wavefront's pieces are in memory
  __syncthreads();
  if (threadIdx.x == 0) *lds = __hip_atomic_fetch_add(&pt.arrived[first], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*lds + 1u != (uint32_t)it.splits) return;
  const int row = threadIdx.x >> 4, part = threadIdx.x & 15, r = it.tile * cut.rows + row;
  if (threadIdx.x == 0) __hip_atomic_store(&pt.arrived[first], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (r >= it.seg.rows) return;
  constexpr int PER = D / 16, BATCH = 4;                   // elements of a thread, pieces at once
  float v[PER], m = -INFINITY, z = 0.f;
#pragma unroll
  for (int x = 0; x < PER; ++x) v[x] = 0.f;
  for (int s0 = 0; s0 < it.splits; s0 += BATCH) {
    float2 mz[BATCH];
    float2 o[BATCH][PER / 2];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int64_t slot = first + row + (int64_t)min(s0 + u, it.splits - 1) * it.seg.rows;
      mz[u] = load_through((const float*)(pt.mz + slot));
#pragma unroll
      for (int x = 0; x < PER / 2; ++x) o[u][x] = load_through(pt.o + slot * D + part * PER + 2 * x);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (s0 + u < it.splits) top = fmaxf(top, mz[u].x);
    const float by = top == -INFINITY ? 1.f : exp2_fast(m - top);
    m = top;
    z *= by;
#pragma unroll
    for (int x = 0; x < PER; ++x) v[x] *= by;
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      if (s0 + u >= it.splits) continue;
      const float w = m == -INFINITY ? 1.f : exp2_fast(mz[u].x - m);
      z += mz[u].y * w;
#pragma unroll
      for (int x = 0; x < PER; ++x) v[x] += (x % 2 == 0 ? o[u][x / 2].x : o[u][x / 2].y) * w;
    }
  }
  Item whole = it;
  whole.slot = -1;
  constexpr int CNT = PER >= 8 ? 8 : 4;
#pragma unroll
  for (int x0 = 0; x0 < PER; x0 += CNT) {
    float y[CNT];
#pragma unroll
    for (int x = 0; x < CNT; ++x) y[x] = v[x0 + x];
    write_row<T, CNT>(a, whole, pt, D, r, part * PER + x0, y, m, z);
  }
}

// What the wavefronts of a split item leave for each other.
template <int D>
struct SplitLds {
  float o[kWaves][16][D + 4];              // padded rows
  float m[kWaves][16], z[kWaves][16];
};

template <typename T, int D, int MT, bool PAD, bool SHARED, bool STREAM>
__device__ __forceinline__ void split_item(const AttendArgs& a, const AttendCut& cut, const Partials& pt, int item, char* lds) {
  typedef Block<T, D> B;
  SplitLds<D>& l = *(SplitLds<D>*)lds;
  Item it;
  if (!find_item<SHARED>(a, cut, item, pt, &it)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const Source src = source_of(a, it);
  int t0, t1;
  tiles_of<SHARED>(a, it, cut.rows, &t0, &t1);
  constexpr int STEP = kWaves * B::KEYS;
  int key = t0 * kKeyTile + wave * B::KEYS;
  PageWindow<B::SUB, STEP> window;                         // (ahead of the queries and limits, which wait for loads of their own)
  if (t0 < t1) window.start(src, key);
  Rows<T, D, MT> rows;
  rows.clear();
  const int all = SHARED ? least_limit(a, it.seg) : 0;
  uint32_t least = 0x7fffffffu, most = 0;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = it.tile * cut.rows + 16 * mt + r16;
    const bool in = r < it.seg.rows;
    rows.lim[mt] = in ? row_limit<SHARED>(a, it.seg, r, all) : 0;
    least = min(least, in ? (uint32_t)rows.lim[mt] : 0x7fffffffu);
    most = max(most, (uint32_t)rows.lim[mt]);
    const int i = (int)((uint32_t)r / (uint32_t)a.G);
    const T* q = (const T*)a.q + (int64_t)(it.seg.c0 + i) * a.qt + (int64_t)(it.h * a.G + (r - i * a.G)) * a.qh;
#pragma unroll
    for (int p = 0; p < B::KP; ++p) {
      const int e = (p * 64 + g * 16) / (int)sizeof(T);
      rows.q[mt][p] = in && e < a.d ? *(const Piece*)(q + e) : Piece{0, 0, 0, 0};
    }
  }
  least = wave_min(least);
  most = wave_max(most);
  const int end = min(t1 * kKeyTile, (int)most);
  const float scale = a.scale * kLog2e;
  bool bad = false;
  auto whole = [&](const Block<T, D>& b) { return b.ok[0] && b.ok[B::SUB - 1]; };
  int block = 0;
  // blocks that every row sees, the next one on its way while one is worked on
  if (key + B::KEYS <= min(end, (int)least)) {
    Block<T, D> cur, nxt;
    load_block<T, D, PAD, STREAM>(cur, src, window, block, key);
    while (whole(cur)) {
      const bool more = key + STEP + B::KEYS <= min(end, (int)least);
      if (more) load_block<T, D, PAD, STREAM>(nxt, src, window, block + 1, key + STEP);
      rows.template step<false>(cur, key, (int)least, (int)most, scale);
      key += STEP;
      window.move(src, ++block);
      if (!more) break;
      cur = nxt;
    }
  }
  // the last ones, and all from a page number out of range on
  const int from = key;
  while (key < end) {
    Block<T, D> b;
    load_block<T, D, PAD, STREAM>(b, src, window, block, key);
    bad = bad || !whole(b);
    rows.template step<true>(b, key, (int)least, (int)most, scale);
    key += STEP;
    window.move(src, ++block);
  }
  if (__any(rows.odd != 0)) rows.template add_odd<false>(src, from, STEP, end, (int)most);
  if (bad && lane == 0) paged_fault(a.map);
  // the wavefronts' results are joined, 16 threads a row
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    if (mt > 0) __syncthreads();
    const float z = sum_over_g(rows.z[mt]);
    if (g == 0) {
      l.m[wave][r16] = rows.m[mt];
      l.z[wave][r16] = z;
    }
#pragma unroll
    for (int hf = 0; hf < B::HN; ++hf)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < B::CW; e += 4)
          *(f32x4*)&l.o[wave][r16][16 * B::CW * hf + B::CW * (4 * g + i) + e] =
              f32x4{rows.o[mt][hf * B::CW + e][i], rows.o[mt][hf * B::CW + e + 1][i], rows.o[mt][hf * B::CW + e + 2][i],
                    rows.o[mt][hf * B::CW + e + 3][i]};
    __syncthreads();
    const int row = threadIdx.x >> 4, part = threadIdx.x & 15, r = it.tile * cut.rows + 16 * mt + row;
    if (r < it.seg.rows) {
      float m = l.m[0][row];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) m = fmaxf(m, l.m[w][row]);
      float by[kWaves], total = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        by[w] = m == -INFINITY ? 1.f : exp2_fast(l.m[w][row] - m);
        total += l.z[w][row] * by[w];
      }
      constexpr int CNT = D / 16 >= 8 ? 8 : 4;
#pragma unroll
      for (int e0 = 0; e0 < D / 16; e0 += CNT) {
        float v[CNT];
        const int at = part * CNT + e0 * 16;
#pragma unroll
        for (int x = 0; x < CNT; ++x) {
          v[x] = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) v[x] += l.o[w][row][at + x] * by[w];
        }
        write_row<T, CNT>(a, it, pt, D, r, at, v, m, total);
      }
    }
  }
  if (!SHARED && pt.arrived != nullptr && it.slot >= 0) join_last<T, D>(a, cut, pt, it, (uint32_t*)&l.m[0][0]);
}

// ------------------------------------------------------------------------------------------------------------------
// Many rows.  bf16.  A tile of 64 keys in LDS: of K the operands (subtile t, piece p, lane), of V the rows, piece c of key k at
// c ^ v_swap(k).  A transposing read takes 32 bytes of each of 16 keys' rows, four keys at a time; the exchange puts those of
// four neighbouring keys into different quarters of 128 bytes.

template <int D>
struct TileBuffer {
  Piece k[kKeyTile / 16][D / 32][64];
  Piece v[kKeyTile][D / 8];
};

template <int D>
__device__ __forceinline__ int v_swap(int key) { return 2 * (key & (D >= 128 ? 7 : 3)); }

// Sends for a tile, straight to LDS: wavefront w has the 16 keys of subtile w.  (The hardware puts lane i's 16 bytes at the given
// place + 16 i.)  Bit t of the result: subtile t's page number is in range; page 0 stands in for one that is not.
template <int D, bool PAD>
__device__ __forceinline__ uint32_t fetch_tile(TileBuffer<D>& to, const Source& s, const PageWindow<4, kKeyTile>& window, int block,
                                               int key0) {
  typedef const __attribute__((address_space(1))) void* Global;
  typedef __attribute__((address_space(3))) void* Lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  uint32_t ok = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) ok |= ((uint32_t)window.page(block, t) < (uint32_t)s.n_pages ? 1u : 0u) << t;
  const int page = ((ok >> wave) & 1u) != 0 ? window.page(block, wave) : 0;
  const int64_t off = (int64_t)page * s.page + (int64_t)(min(key0 + 16 * wave, s.last) & (s.ps - 1)) * s.tok;
  const char* kb = uniform(s.k + off);
  const uint32_t ko = (uint32_t)r * (uint32_t)s.tok + (uint32_t)g * 16u;
#pragma unroll
  for (int p = 0; p < D / 32; ++p) {
    const bool in = !PAD || p * 64 + g * 16 < s.d * 2;     // beyond d: the row's first piece (read as zeros)
    __builtin_amdgcn_global_load_lds((Global)(uniform(kb + (PAD ? 0 : p * 64)) + offset(!PAD ? ko : in ? ko + p * 64u : ko - g * 16u)),
                                     (Lds)&to.k[wave][p][0], 16, 0, 0);
  }
  constexpr int PR = D / 8, RPI = 64 / PR;                 // pieces of a row, rows of an instruction
#pragma unroll
  for (int i = 0; i < 16 / RPI; ++i) {
    const int piece = (lane % PR) ^ v_swap<D>(i * RPI + lane / PR);
    const uint32_t vo = (uint32_t)(lane / PR) * (uint32_t)s.tok + (!PAD || piece * 8 < s.d ? (uint32_t)piece * 16u : 0u);
    __builtin_amdgcn_global_load_lds((Global)(uniform(s.v + off + (int64_t)i * RPI * s.tok) + offset(vo)), (Lds)&to.v[16 * wave + i * RPI][0], 16, 0, 0);
  }
  return ok;
}

// A wavefront's step over a tile in LDS.  MASKED: some row may not see some key, or its reference may have to move.  Else every row
// sees every key and no reference moves; returns false, nothing done, if one has to.  (A branch that rescales the accumulators
// makes the compiler keep them twice, which does not fit the registers: the prefill chunk took 1629 us with it and 1142 without.)
template <int D, int MT, bool PAD, bool MASKED>
__device__ __forceinline__ bool tile_step(Rows<__bf16, D, MT>& R, const TileBuffer<D>& b, int key0, uint32_t ok, int least, int most,
                                          int d, float scale) {
  typedef Block<__bf16, D> B;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  // Reads from LDS are a step ahead of the products that take them, and held there: left alone the scheduler gathers more of them
  // than there are registers for.
  f32x4 x[MT][4];
  Piece kf[2][B::KP];
  auto read_k = [&](int t) {
#pragma unroll
    for (int p = 0; p < B::KP; ++p) kf[t & 1][p] = b.k[t][p][lane];
  };
  read_k(0);
  __builtin_amdgcn_s_setprio(1);                           // products before the other wavefronts' softmax: 1106 us, 1084 so
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if (t < 3) read_k(t + 1);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x[mt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < B::KP; ++p) {
      Piece k = kf[t & 1][p];
      if (PAD && p * 32 + g * 8 >= d) k = Piece{0, 0, 0, 0};
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        x[mt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, R.q[mt][p]),
                                                           x[mt][t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  // V: lanes 4 j + c of 16 name columns 4 c .. 4 c + 3 of key j, lane i gets column i of the four keys
  typedef short Half4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) Half4* LdsHalf4;
  union Values { Half4 h[2]; uint32_t u[4]; bf16x8 v; };
  constexpr int STEPS = 2 * B::NT, AHEAD = 2;
  Values vf[AHEAD + 1];
  const uint32_t swap = offset((uint32_t)(v_swap<D>(4 * g + (r >> 2)) ^ ((r >> 1) & 1)) << 4);
  const char* vrow = (const char*)&b.v[4 * g + (r >> 2)][0] + (r & 1) * 8;
  auto read_v = [&](int i) {
    const int hb = i / B::NT, nt = i % B::NT;
    const char* at = vrow + ((uint32_t)(nt << 5) ^ swap);
    vf[i % (AHEAD + 1)].h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf4)(at + (32 * hb) * (D * 2)));
    vf[i % (AHEAD + 1)].h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf4)(at + (32 * hb + 16) * (D * 2)));
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) read_v(i);
  Weights<__bf16> w[2][MT];
  float tops[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (MASKED) x[mt][t][i] = ((ok >> t) & 1u) != 0 && key0 + 16 * t + 4 * g + i < R.lim[mt] ? x[mt][t][i] : -INFINITY;
        top = fmaxf(top, x[mt][t][i]);
      }
    tops[mt] = top * scale;
  }
  if (MASKED) {
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      if (__any(tops[mt] > R.m[mt] + kSlack)) {
        const float to = fmaxf(R.m[mt], max_over_g(tops[mt]));
        const float by = to == -INFINITY ? 1.f : exp2_fast(R.m[mt] - to);
        R.m[mt] = to;
        R.z[mt] *= by;
#pragma unroll
        for (int t = 0; t < B::NT; ++t) R.o[mt][t] *= by;
      }
  } else {
    bool rises = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) rises = rises || tops[mt] > R.m[mt] + kWideSlack;
    if (__any(rises)) return false;
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const float base = R.m[mt] == -INFINITY ? 0.f : R.m[mt];
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      float p[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[t][i] = exp2_fast(__builtin_fmaf(x[mt][2 * hb + t][i], scale, -base));
          R.z[mt] += p[t][i];
        }
      w[hb][mt].set(p);
    }
  }
  uint32_t seen[2][4];                                     // of the two keys of each word, those that any of the rows sees
  if (MASKED) {
#pragma unroll
    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int key = key0 + 32 * hb + B::v_key(2 * p, g);
        const bool in = ((ok >> (2 * hb + (p >> 1))) & 1u) != 0;
        seen[hb][p] = (in && key < most ? 0xffffu : 0u) | (in && key + 1 < most ? 0xffff0000u : 0u);
      }
  }
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int hb = i / B::NT, nt = i % B::NT;
    if (i + AHEAD < STEPS) read_v(i + AHEAD);
    Values& y = vf[i % (AHEAD + 1)];
    if (MASKED) {                                          // as in Rows::add
      const bool differ = least < most;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        y.u[p] &= seen[hb][p];
        if (differ) {
          const uint32_t bits = not_finite<__bf16>(y.u[p]);
          R.odd |= bits;
          y.u[p] &= ~whole_elements<__bf16>(bits);
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
      R.o[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y.v, w[hb][mt].w, R.o[mt][nt], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  return true;
}

template <int D, int MT, bool PAD, bool SHARED>
__device__ __forceinline__ void tile_item(const AttendArgs& a, const AttendCut& cut, const Partials& pt, int item, char* lds) {
  typedef Block<__bf16, D> B;
  TileBuffer<D>* buf = (TileBuffer<D>*)lds;
  Item it;
  if (!find_item<SHARED>(a, cut, item, pt, &it)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int row0 = it.tile * cut.rows + wave * 16 * MT;
  const Source src = source_of(a, it);
  int t0, t1;
  tiles_of<SHARED>(a, it, cut.rows, &t0, &t1);
  PageWindow<4, kKeyTile> window;                          // (ahead of the queries and limits, which wait for loads of their own)
  if (t0 < t1) window.start(src, t0 * kKeyTile);
  Rows<__bf16, D, MT> rows;
  rows.clear();
  const int all = SHARED ? least_limit(a, it.seg) : 0;
  uint32_t least = 0x7fffffffu, most = 0;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row0 + 16 * mt + r16;
    const bool in = r < it.seg.rows;
    rows.lim[mt] = in ? row_limit<SHARED>(a, it.seg, r, all) : 0;
    if (!in) rows.m[mt] = 0.f;                             // rows that are not there have logits 0: no reference to move for them
    least = min(least, in ? (uint32_t)rows.lim[mt] : 0x7fffffffu);
    most = max(most, (uint32_t)rows.lim[mt]);
    const int i = (int)((uint32_t)r / (uint32_t)a.G);
    const __bf16* q = (const __bf16*)a.q + (int64_t)(it.seg.c0 + i) * a.qt + (int64_t)(it.h * a.G + (r - i * a.G)) * a.qh;
#pragma unroll
    for (int p = 0; p < B::KP; ++p) {
      const int e = p * 32 + g * 8;
      rows.q[mt][p] = in && e < a.d ? *(const Piece*)(q + e) : Piece{0, 0, 0, 0};
    }
  }
  least = wave_min(least);
  most = wave_max(most);
  // keys that all rows of the workgroup see (an own segment's limits rise with the row)
  const int all_see = SHARED ? all : row_limit<SHARED>(a, it.seg, it.tile * cut.rows, 0);
  const float scale = a.scale * kLog2e;
  bool bad = false;
  if (t0 < t1) {
    uint32_t ok = fetch_tile<D, PAD>(buf[0], src, window, 0, t0 * kKeyTile);
    int t = t0;
    // tile t's pieces have landed, everybody's after the barrier, behind which nobody reads the other buffer any more: the next go there
    auto next = [&]() {
      __builtin_amdgcn_s_waitcnt(0x0070);                  // vmcnt 0, lgkmcnt 0
      __syncthreads();
      const uint32_t here = ok;
      if (t + 1 < t1) ok = fetch_tile<D, PAD>(buf[(t + 1 - t0) & 1], src, window, t + 1 - t0, (t + 1) * kKeyTile);
      return here;
    };
    bool fetched = false;                                  // tile t has been waited for
    uint32_t here = 0;
    const int from = t0 * kKeyTile;
    while (most == 0 && t < t1) {                          // a wavefront without rows only fetches
      next();
      ++t;
      window.move(src, t - t0);
    }
    while (t < t1) {
      if (!fetched) here = next();
      const int key0 = t * kKeyTile;
      bad = bad || here != 15u;
      if (key0 < (int)most)
        tile_step<D, MT, PAD, true>(rows, buf[(t - t0) & 1], key0, here, (int)least, (int)most, a.d, scale);
      fetched = false;
      ++t;
      window.move(src, t - t0);
      // tiles that every row sees, as long as no reference has to move.  (Wavefronts may leave at different tiles: next() has the barriers,
      // one a tile.)
      while (t < t1 && ok == 15u && (t + 1) * kKeyTile <= all_see) {
        here = next();
        fetched = !tile_step<D, MT, PAD, false>(rows, buf[(t - t0) & 1], t * kKeyTile, 15u, (int)least, (int)most, a.d, scale);
        if (fetched) break;
        ++t;
        window.move(src, t - t0);
      }
    }
    if (__any(rows.odd != 0))
      rows.template add_odd<true>(src, from, B::KEYS, min(t1 * kKeyTile, (int)most), (int)most);
  }
  if (bad && lane == 0) paged_fault(a.map);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int r = row0 + 16 * mt + r16;
    const float z = sum_over_g(rows.z[mt]);
    if (r >= it.seg.rows) continue;
#pragma unroll
    for (int nt = 0; nt < B::NT; ++nt) {
      const float v[4] = {rows.o[mt][nt][0], rows.o[mt][nt][1], rows.o[mt][nt][2], rows.o[mt][nt][3]};
      write_row<__bf16, 4>(a, it, pt, D, r, 16 * nt + 4 * g, v, rows.m[mt], z);
    }
  }
}

// ------------------------------------------------------------------------------------------------------------------
// Joins the pieces of rows that were cut: NW wavefronts a row, each 4 D bytes' lanes of them every so many-th piece, four at a time,
// with a running maximum of their references; then lanes and wavefronts are joined.  One pass: what it costs is the latency of the
// loads that depend on each other (the sequence, its plan, the pieces).
template <typename T, int D, int NW>
__device__ __forceinline__ void join_row(const AttendArgs& a, const Partials& own, const Partials& shared, int64_t row, float* so_, float* sm,
                                         float* sz) {
  constexpr int LPP = D / 4;                               // lanes of a piece, four elements each
  constexpr int PPW = 64 / LPP;                            // pieces that a wavefront takes at once
  float (*so)[D] = (float (*)[D])so_;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tok = (int)(row / a.Hq), hq = (int)(row - (int64_t)tok * a.Hq), h = hq / a.G;
  const int b = sequence_by_wave(a.cu_q, a.n_seqs, tok);
  const int4 p = own.plan[b];
  const int g = a.n_groups > 0 ? own.group[b] : -1;
  const int r = (tok - p.x) * a.G + hq - h * a.G;
  if (p.z <= 0 || tok < p.x || r >= p.y) return;           // written whole
  int n1 = 0;
  int64_t at1 = 0;
  int rows1 = 0;
  if (g >= 0) {
    const int4 q = shared.plan[g];
    const int rs = (tok - q.x) * a.G + hq - h * a.G;
    if (q.z > 0 && tok >= q.x && rs < q.y) {
      n1 = q.z;
      rows1 = q.y;
      at1 = (int64_t)(uint32_t)q.w + (int64_t)h * q.z * q.y + rs;
    }
  }
  const int n0 = p.z, total = n0 + n1;
  const int64_t at0 = (int64_t)(uint32_t)p.w + (int64_t)h * p.z * p.y + r;
  const int sub = lane / LPP, e = (lane % LPP) * 4;
  float m = -INFINITY, z = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = (wave % NW) * PPW + sub; i0 < total; i0 += 4 * NW * PPW) {
    float2 mz[4];
    f32x4 o[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = min(i0 + u * NW * PPW, total - 1);     // past the end: the last one again, not counted
      const Partials& f = i < n0 ? own : shared;
      const int64_t s = i < n0 ? at0 + (int64_t)i * p.y : at1 + (int64_t)(i - n0) * rows1;
      mz[u] = f.mz[s];
      o[u] = *(const f32x4*)(f.o + s * D + e);
    }
    float top = m;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * NW * PPW < total) top = fmaxf(top, mz[u].x);
    const float by = top == -INFINITY ? 1.f : exp2_fast(m - top);
    m = top;
    z *= by;
    acc *= by;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * NW * PPW < total) {
        const float w = m == -INFINITY ? 1.f : exp2_fast(mz[u].x - m);
        z += mz[u].y * w;
        acc += o[u] * w;
      }
  }
#pragma unroll
  for (int x = LPP; x < 64; x *= 2) {                      // the wavefront's lanes that have the same elements
    const float m2 = __shfl_xor(m, x), z2 = __shfl_xor(z, x);
    const float top = fmaxf(m, m2), by = top == -INFINITY ? 1.f : exp2_fast(m - top), by2 = top == -INFINITY ? 1.f : exp2_fast(m2 - top);
    m = top;
    z = z * by + z2 * by2;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] = acc[c] * by + __shfl_xor(acc[c], x) * by2;
  }
  if (NW > 1) {
    if (lane < LPP) *(f32x4*)&so[wave][e] = acc;
    if (lane == 0) {
      sm[wave] = m;
      sz[wave] = z;
    }
    __syncthreads();
    if (wave % NW != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, sm[wave + w]);
    m = top;
    z = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float by = m == -INFINITY ? 1.f : exp2_fast(sm[wave + w] - m);
      z += sz[wave + w] * by;
      acc += *(const f32x4*)&so[wave + w][e] * by;
    }
  }
  if (lane < LPP && e < a.d) {
    const float by = z == 0.f ? 0.f : 1.f / z;
    typedef T Out __attribute__((ext_vector_type(4)));
    *(Out*)((T*)a.out + (int64_t)tok * a.ot + (int64_t)hq * a.oh + e) =
        Out{(T)(acc[0] * by), (T)(acc[1] * by), (T)(acc[2] * by), (T)(acc[3] * by)};
  }
  if (lane == 0 && a.lse != nullptr) a.lse[(int64_t)hq * a.total_q + tok] = z == 0.f ? -INFINITY : (m + __log2f(z)) * kLn2;
}

// The rows in turn; nothing where no row was cut.  With several wavefronts a row there is a workgroup for each row (a barrier in the way of
// a second one).
template <typename T, int D, int NW>
__global__ void __launch_bounds__(NW > kWaves ? NW * 64 : kThreads) attend_join_kernel(AttendArgs a, Partials own, Partials shared) {
  constexpr int WAVES = NW > kWaves ? NW : kWaves;
  __shared__ __attribute__((aligned(16))) float so[WAVES * D];
  __shared__ float sm[WAVES], sz[WAVES];
  if (*own.cut == 0) return;
  if constexpr (NW > 1) {
    static_assert(NW == WAVES, "a workgroup has one row");
    join_row<T, D, NW>(a, own, shared, (int64_t)blockIdx.x, so, sm, sz);
  } else {
    for (int64_t row = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6); row < (int64_t)a.total_q * a.Hq; row += (int64_t)gridDim.x * WAVES)
      join_row<T, D, 1>(a, own, shared, row, so, sm, sz);
  }
}

// ------------------------------------------------------------------------------------------------------------------
template <typename T, int D, int KIND, bool PAD, bool SHARED, bool STREAM>
__device__ __forceinline__ void run_item(const AttendArgs& a, const AttendCut& cut, const Partials& pt, int item, char* lds) {
  if constexpr (KIND == kSplit) split_item<T, D, 1, PAD, SHARED, STREAM>(a, cut, pt, item, lds);
  if constexpr (KIND == kTile1) tile_item<D, 1, PAD, SHARED>(a, cut, pt, item, lds);
  if constexpr (KIND == kTile2) tile_item<D, 2, PAD, SHARED>(a, cut, pt, item, lds);
}
template <int D, int KIND>
constexpr size_t lds_of() {
  return KIND == kNone ? 0 : KIND == kSplit ? sizeof(SplitLds<D>) : 2 * sizeof(TileBuffer<D>);
}

// One launch has the items of both kinds, the shared ones first: those are the longer ones, and the own ones fill the units as they
// come free.  (In turn, eight of each, some units end up with more of the long ones: shared prompt 121 us, 93 so.)
template <typename T, int D, int OWN, int SHARED, bool PAD, bool STREAM>
__global__ void __launch_bounds__(kThreads, D > 128 ? 1 : 2)
attend_kernel(AttendArgs a, AttendCut own, AttendCut shared, Partials po, Partials ps, int n_shared) {
  constexpr size_t LDS = lds_of<D, OWN>() > lds_of<D, SHARED>() ? lds_of<D, OWN>() : lds_of<D, SHARED>();
  __shared__ __attribute__((aligned(16))) char lds[LDS];
  int i = (int)blockIdx.x;
  if constexpr (SHARED != kNone) {
    if (i < n_shared) {
      run_item<T, D, SHARED, PAD, true, STREAM>(a, shared, ps, i, lds);
      return;
    }
    i -= n_shared;                                         // a multiple of 8: an item's die is its head's
  }
  run_item<T, D, OWN, PAD, false, STREAM>(a, own, po, i, lds);
}

template <typename T, int D, int OWN, int SHARED, bool STREAM>
hipError_t launch_kinds(const AttendArgs& a, const AttendCut& own, const AttendCut& shared, const Partials& po, const Partials& ps,
                        hipStream_t st) {
  const int64_t rows = (int64_t)a.total_q * a.G;
  const int64_t n_own = (max_items(own, rows, a.n_seqs, a.Hk) + 7) & ~int64_t(7);
  const int64_t n_shared = SHARED == kNone ? 0 : (max_items(shared, rows, a.n_groups, a.Hk) + 7) & ~int64_t(7);
  if (n_own + n_shared >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(n_own + n_shared)), block(kThreads);
  if (a.d == D)
    hipLaunchKernelGGL((attend_kernel<T, D, OWN, SHARED, false, STREAM>), grid, block, 0, st, a, own, shared, po, ps, (int)n_shared);
  else
    hipLaunchKernelGGL((attend_kernel<T, D, OWN, SHARED, true, STREAM>), grid, block, 0, st, a, own, shared, po, ps, (int)n_shared);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const PagedWorkspace& ws, const AttendArgs& args, hipStream_t st) {
  AttendArgs a = args;
  constexpr bool kTiles = sizeof(T) == 2 && D <= 128;
  const AttendRule rule = rule_for(kTiles, a.total_q, a.G, a.Hk, a.n_seqs, a.n_groups, a.max_q_len, a.max_kv_len, a.key_bytes, ws.part_rows);
  const AttendCut own = rule.own, shared = rule.shared;
  if (!rule.groups) a.n_groups = 0;
  Partials po, ps;
  ps.o = ws.part;
  ps.mz = ws.part_mz;
  ps.plan = ws.plan + kPagedMaxSeqs;
  ps.group = nullptr;
  po.o = ws.part + shared.cap * D;
  po.mz = ws.part_mz + shared.cap;
  po.plan = ws.plan;
  po.group = ws.group;
  po.cut = ps.cut = ws.cut;
  ps.arrived = nullptr;
  po.arrived = rule.joined ? ws.arrived + shared.cap : nullptr;
  hipError_t e = hipErrorInvalidValue;
  const int ks = a.n_groups > 0 ? shared.rows : kNone;
  const bool once = rule.most <= kSplit;                   // a sequence's keys are read by one tile of rows
  if constexpr (kTiles) {
    if (ks == kNone) {
      e = own.rows == kTile2   ? launch_kinds<T, D, kTile2, kNone, true>(a, own, shared, po, ps, st)
          : own.rows == kTile1 ? launch_kinds<T, D, kTile1, kNone, true>(a, own, shared, po, ps, st)
          : once               ? launch_kinds<T, D, kSplit, kNone, true>(a, own, shared, po, ps, st)
                               : launch_kinds<T, D, kSplit, kNone, false>(a, own, shared, po, ps, st);
    } else if (own.rows == kTile1) {
      e = ks == kTile2   ? launch_kinds<T, D, kTile1, kTile2, true>(a, own, shared, po, ps, st)
          : ks == kTile1 ? launch_kinds<T, D, kTile1, kTile1, true>(a, own, shared, po, ps, st)
                         : launch_kinds<T, D, kTile1, kSplit, true>(a, own, shared, po, ps, st);
    } else {
      e = ks == kTile2   ? launch_kinds<T, D, kSplit, kTile2, true>(a, own, shared, po, ps, st)
          : ks == kTile1 ? launch_kinds<T, D, kSplit, kTile1, true>(a, own, shared, po, ps, st)
                         : launch_kinds<T, D, kSplit, kSplit, false>(a, own, shared, po, ps, st);
    }
  } else if (ks == kNone) {
    e = once ? launch_kinds<T, D, kSplit, kNone, true>(a, own, shared, po, ps, st)
             : launch_kinds<T, D, kSplit, kNone, false>(a, own, shared, po, ps, st);
  } else {
    e = launch_kinds<T, D, kSplit, kSplit, false>(a, own, shared, po, ps, st);
  }
  if (e != hipSuccess || po.arrived != nullptr) return e;
  const int64_t out_rows = (int64_t)a.total_q * a.Hq;
  // few rows are cut into many pieces each
  if (out_rows <= 256)
    hipLaunchKernelGGL((attend_join_kernel<T, D, 16>), dim3((unsigned)out_rows), dim3(1024), 0, st, a, po, ps);
  else if (out_rows <= 2048)
    hipLaunchKernelGGL((attend_join_kernel<T, D, kWaves>), dim3((unsigned)out_rows), dim3(kThreads), 0, st, a, po, ps);
  else
    hipLaunchKernelGGL((attend_join_kernel<T, D, 1>), dim3((unsigned)(out_rows < 4096 * kWaves ? (out_rows + kWaves - 1) / kWaves : 4096)),
                       dim3(kThreads), 0, st, a, po, ps);
  return hipGetLastError();
}

}  // namespace

}  // namespace asl
