// Tile items of drafted trees (bf16, d <= 128): 128 rows whose keys come through LDS in steps of 32.  Bound by the keys' way from memory where
// drafts are small, by products and vector work where they are not.  A wavefront has 32 rows, on v_mfma_f32_32x32x16_bf16: beside one of
// those, which takes 32 cycles, four additions and an exponential are free, beside two 16x16x32, which do as much, they take 20 more
// (measured on loops of nothing else).  For that it does three things at once that do not wait for each other: the logits of step t + 1, the
// exponentials of step t, the products of step t - 1 with its values.  Keys are sent for three steps ahead, values two, so that two steps'
// are always on their way.
// 32 sequences of 2300 keys, 16 to 32 nodes, 8 heads, d = 128: 73 us; the steps run at 5.5 TB/s, but an item takes 10 us to begin (page numbers,
// queries, parents, first keys: loads that depend on each other) and end.  60 nodes of 28 heads on 131089 keys: 159 us = 712 TFLOP/s, 1800 cycles
// for a step of both workgroups of a unit, where products take 1024 and LDS reads 1280.  With 16x16x32 products and tiles of 64 keys: 120 and 171.
//
//   x^T = K Q^T: lane (r = lane % 32, h = lane / 32) holds K[r][16 c + 8 h ..]; its accumulator has row r and keys 8 j + 4 h .. + 3, j < 4;
//   out^T += V^T P^T: contraction slot (h, e) = key 16 u + 8 (e / 4) + 4 h + e % 4, u < 2, so that a lane's probabilities are the
//   operand where they stand.
#pragma once
#include "attend_body.h"

namespace asl {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kStep = 32;

// Rings of four steps: K by 16 keys and 64 bytes of their rows, a lane's 16 bytes behind the other; V by rows with their pieces exchanged:
// piece c of key k at c ^ step_swap(k), so that the 32 lanes that a transposing read serves at once, 64 bytes of each of four keys, fall
// into different banks.
template <int D>
struct StepRing {
  Piece k[4][kStep / 16][D / 32][64];
  Piece v[4][kStep][D / 8];
};
// Loads of a wavefront for a step's keys, and as many for its values.
template <int D> constexpr int kStepLoads = D / 64;

template <int D>
__device__ __forceinline__ int step_swap(int key) { return D >= 128 ? 2 * (2 * (key & 3) + ((key >> 2) & 1)) : 2 * (key & 2); }

// Where the steps' subtiles stand in the pages, bytes from the head's first on: of 32 steps a lane each, with the page numbers of the 32 behind
// them on their way.  Page 0 stands in for a number out of range; `good` has the bits of those that are in range, `before` those of the 32 steps
// before, and `bad` is the first step of all so far that has one that is not.
struct StepWindow {
  static constexpr int kSteps = 32;
  uint32_t lo, hi;
  int next, key, first, bad;
  uint64_t good, before;

  __device__ __forceinline__ int subtile(const Source& s, int step) const {      // the lane's key; behind the end the last subtile's
    const int lane = threadIdx.x & 63;
    return min(key + (step + (lane >> 1)) * kStep + 16 * (lane & 1), s.last);
  }
  __device__ __forceinline__ void take(const Source& s, int number) {
    const bool in = (uint32_t)number < (uint32_t)s.n_pages;
    const int64_t place = (int64_t)(in ? number : 0) * s.page + (int64_t)(subtile(s, first) & (s.ps - 1)) * s.tok;
    lo = (uint32_t)place;
    hi = (uint32_t)((uint64_t)place >> 32);
    before = good;
    good = __ballot(in);
    if (~good != 0) bad = min(bad, first + (int)__builtin_ctzll(~good) / 2);
    next = s.table[subtile(s, first + kSteps) >> s.shift];
  }
  __device__ __forceinline__ void start(const Source& s, int key0, int number) {
    key = key0;
    first = 0;
    bad = 0x7fffffff;
    good = 0;
    take(s, number);
  }
  __device__ __forceinline__ int64_t place(const Source& s, int step, int sub) {
    if (step - first >= kSteps) {
      first += kSteps;
      take(s, next);
    }
    const int l = 2 * (step - first) + sub;
    return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, l));
  }
  // Of the two subtiles of a step, at most three behind the last one sent for, those in range.
  __device__ __forceinline__ uint32_t in_range(int step) const {
    return (uint32_t)(step >= first ? good >> (2 * (step - first)) : before >> (2 * (step - first + kSteps))) & 3u;
  }
};

// Sends 16 bytes a lane from base + offset straight to LDS, lane i's to `to` + 16 i.  Not the builtin: beside it the compiler has every
// transposing read of LDS wait for all sends, and here two steps' are always on their way; step_item has the waits.  (It has no
// register to write, and the compiler's own waits count it as nothing, so that they are longer than they need be.)
__device__ __forceinline__ void send_to_lds(uint32_t to, const char* base, uint32_t offset) {
  const uint32_t m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)to);
  uint32_t kept;                                           // (the compiler's m0, which no clobber can name)
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
               : "=&s"(kept)
               : "s"(m0), "v"(offset), "s"(uniform(base))
               : "memory");
}

// The same if `on` is not 0.  (A branch that the compiler knew of would cut the products beside it into pieces, which it then keeps
// registers of twice: 300 of them in memory.)
__device__ __forceinline__ void send_to_lds_if(uint32_t on, uint32_t to, const char* base, uint32_t offset) {
  const uint32_t m0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)to), cond = (uint32_t)__builtin_amdgcn_readfirstlane((int)on);
  uint32_t kept;
  asm volatile("s_cmp_eq_u32 %4, 0\n\ts_cbranch_scc1 .Lskip%=\n\ts_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
               "global_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0\n.Lskip%=:"
               : "=&s"(kept)
               : "s"(m0), "v"(offset), "s"(uniform(base)), "s"(cond)
               : "memory", "scc");
}

// A lane's offsets in its wavefront's part of a step: half of the pieces of 16 keys, and 8 rows of values.
template <int D>
struct StepLane {
  uint32_t k[kStepLoads<D>], v[kStepLoads<D>];

  template <bool PAD>
  __device__ __forceinline__ void set(const Source& s, int wave) {
    const int lane = threadIdx.x & 63;
    constexpr int PR = D / 8, RPI = 64 / PR;               // pieces of a row, rows of an instruction
#pragma unroll
    for (int i = 0; i < kStepLoads<D>; ++i) {
      const int piece = 4 * ((wave & 1) * kStepLoads<D> + i) + (lane >> 4);
      k[i] = (uint32_t)(lane & 15) * (uint32_t)s.tok + (!PAD || piece * 8 < s.d ? (uint32_t)piece * 16u : 0u);   // beyond d: read as zeros
      const int row = 8 * (wave & 1) + i * RPI + lane / PR, vp = (lane % PR) ^ step_swap<D>(row);
      v[i] = (uint32_t)row * (uint32_t)s.tok + (!PAD || vp * 8 < s.d ? (uint32_t)vp * 16u : 0u);                 // beyond d: of no use
    }
  }
};

// A wavefront's running results for 32 rows, lanes r and r + 32 each the same one.
template <int D, bool DRAFT>
struct StepRows : Sight<1, DRAFT> {
  Piece q[D / 16];
  f32x16 o[D / 32];        // element 32 n + 8 j + 4 h + c of the row in o[n][4 j + c]
  float m, z;              // reference and, of this lane's keys, sum
  int lim;
  uint32_t odd;            // values were left out
};

// A lane's part of a step's 32 logits of its row, and of their probabilities.
struct StepLogits {
  f32x16 x;
};
struct StepWeights {
  bf16x8 w[2];

  __device__ __forceinline__ void set(int u, const float (&p)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[u][e] = (__bf16)p[e];    // (each rounds to 8 bits: see Weights)
  }
};

// 32 keys' 16 elements from 16 c on as an operand.
template <int D, bool PAD>
__device__ __forceinline__ Piece step_key(const StepRing<D>& ring, int block, int c, int d) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  Piece k = ring.k[block & 3][(lane >> 4) & 1][c >> 1][32 * (c & 1) + 16 * h + (lane & 15)];
  if (PAD && 16 * c + 8 * h >= d) k = Piece{0, 0, 0, 0};
  return k;
}

// 16 keys' 32 elements from 32 n on as an operand, turned: of 16 lanes, 4 j + c name columns 4 c .. 4 c + 3 of key j, and lane i gets
// column i of the four keys.
template <int D>
__device__ __forceinline__ Piece step_value(const StepRing<D>& ring, int block, int u, int n) {
  typedef short Half4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) Half4* LdsHalf4;
  union { Half4 half[2]; Piece p; } y;
  const int lane = threadIdx.x & 63, r = lane & 15, key = 4 * (lane >> 5) + (r >> 2);
  const uint32_t piece = (uint32_t)(4 * n) ^ (uint32_t)(step_swap<D>(key) ^ (2 * ((lane >> 4) & 1) + ((r >> 1) & 1)));
  const char* at = (const char*)&ring.v[block & 3][key][0] + piece * 16u + (r & 1) * 8 + 16 * u * (D * 2);
  y.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf4)at);                // (keys 8 on are exchanged as keys 0 on)
  y.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf4)(at + 8 * (D * 2)));
  return y.p;
}

__device__ __forceinline__ f32x16 step_product(Piece a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
}

template <int D, bool PAD, bool DRAFT>
__device__ __forceinline__ void step_logits(const StepRows<D, DRAFT>& R, const StepRing<D>& ring, int block, int d, StepLogits& out) {
#pragma unroll
  for (int i = 0; i < 16; ++i) out.x[i] = 0.f;
#pragma unroll
  for (int c = 0; c < D / 16; ++c) out.x = step_product(step_key<D, PAD>(ring, block, c, d), __builtin_bit_cast(bf16x8, R.q[c]), out.x);
}

__device__ __forceinline__ float step_top(const StepLogits& l) {
  float top = l.x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, l.x[i]);
  return top;
}

// Probability i of a step, for a row whose reference is `base`.
template <int D, bool DRAFT>
__device__ __forceinline__ float step_exp(StepRows<D, DRAFT>& R, const StepLogits& l, int i, float scale, float base) {
  const float p = exp2_fast(__builtin_fmaf(l.x[i], scale, -base));
  R.z += p;
  return p;
}
template <int D, bool DRAFT>
__device__ __forceinline__ void step_weights(StepRows<D, DRAFT>& R, const StepLogits& l, float scale, StepWeights& out) {
  const float base = R.m == -INFINITY ? 0.f : R.m;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = step_exp(R, l, 8 * u + e, scale, base);
    out.set(u, p);
  }
}

template <int D, bool DRAFT>
__device__ __forceinline__ void step_values(StepRows<D, DRAFT>& R, const StepRing<D>& ring, int block, const StepWeights& w) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int n = 0; n < D / 32; ++n) R.o[n] = step_product(step_value<D>(ring, block, u, n), w.w[u], R.o[n]);
}

// A step whose keys not every row may see, or at which a reference may move.  ok: bit t, the page number of keys 16 t on is in range.
template <int D, bool PAD, bool DRAFT>
__device__ __forceinline__ void step_general(StepRows<D, DRAFT>& R, const StepRing<D>& ring, int block, int key0, uint32_t ok, int least, int most,
                                             int d, float scale) {
  const int h = (threadIdx.x & 63) >> 5;
  StepLogits l;
  step_logits<D, PAD>(R, ring, block, d, l);
  const uint32_t there = ((ok & 1u) != 0 ? 0xffffu : 0u) | ((ok & 2u) != 0 ? 0xffff0000u : 0u);
  uint32_t sight;
  if constexpr (DRAFT) sight = R.window(0, R.lim, key0);
  else sight = R.lim - key0 >= 32 ? ~0u : R.lim <= key0 ? 0u : (1u << (R.lim - key0)) - 1u;
  sight &= there;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; ++i) {                           // key 8 (i / 4) + 4 h + i % 4
    l.x[i] = ((sight >> (4 * h)) >> (8 * (i >> 2) + (i & 3)) & 1u) != 0 ? l.x[i] : -INFINITY;
    top = fmaxf(top, l.x[i]);
  }
  top *= scale;
  if (__any(top > R.m + kSlack)) {
    const float to = fmaxf(R.m, fmaxf(top, __shfl_xor(top, 32)));
    const float by = to == -INFINITY ? 1.f : exp2_fast(R.m - to);
    R.m = to;
    R.z *= by;
#pragma unroll
    for (int n = 0; n < D / 32; ++n) R.o[n] *= by;
  }
  StepWeights w;
  step_weights(R, l, scale, w);
  // Probability 0 does not keep a value that is no number out of the sum (see Rows::add): keys that no row sees count as zeros, and where rows
  // differ in what they see, infinities and NaN do too, and are added afterwards for the rows that see them.
  const uint32_t any = there & (most - key0 >= 32 ? ~0u : (1u << (most - key0)) - 1u);     // (most > key0)
  const bool differ = least < most;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    uint32_t seen[4];                                      // of the two keys of each word
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t two = any >> (16 * u + 8 * (p >> 1) + 4 * h + 2 * (p & 1));
      seen[p] = ((two & 1u) != 0 ? 0xffffu : 0u) | ((two & 2u) != 0 ? 0xffff0000u : 0u);
    }
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
      Piece y = step_value<D>(ring, block, u, n);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        y[p] &= seen[p];
        if (differ) {
          const uint32_t bits = not_finite<__bf16>(y[p]);
          R.odd |= bits;
          y[p] &= ~whole_elements<__bf16>(bits);
        }
      }
      R.o[n] = step_product(y, w.w[u], R.o[n]);
    }
  }
  if (__any(R.odd != 0)) {                                 // (rare: key by key)
    R.odd = 0;
#pragma unroll 1
    for (int key = 0; key < kStep; ++key) {
      const bool sees = ((sight >> key) & 1u) != 0;
      const char* row = (const char*)&ring.v[block & 3][key][0];
#pragma unroll
      for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint2 two = *(const uint2*)(row + ((uint32_t)(4 * n + j) ^ (uint32_t)step_swap<D>(key)) * 16u + 8 * h);
          const uint32_t word[2] = {two.x, two.y};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t bits = c & 1 ? word[c >> 1] & 0xffff0000u : word[c >> 1] << 16;
            if (sees && not_finite<__bf16>(bits) != 0) R.o[n][4 * j + c] += __uint_as_float(bits);
          }
        }
    }
  }
}

// Operands from LDS that are on their way.
struct StepAhead {
  static constexpr int N = 4;
  Piece x[N];
};

// The middle of three steps: probabilities of `here` to `now`, beside the products of the step before it with its values and the logits of the
// one behind it.  Nothing of it waits for another part; it is written in the order in which it is to go out: an operand's product, beside it
// a probability and now and then a send, then the read of the fourth operand behind it, the last four of them the next step's first.
// Returns whether some row's reference has to move for the logits of the step behind, which are there before the last products are.
template <int D, bool PAD, bool DRAFT, typename Send>
__device__ __forceinline__ bool step_all(StepRows<D, DRAFT>& R, const StepRing<D>& ring, int block, int d, float scale, const StepLogits& here,
                                         StepLogits& next, const StepWeights& before, StepWeights& now, StepAhead& ahead, Send send) {
  constexpr int NV = D / 16, N = 2 * NV, AH = StepAhead::N;      // products with values, and as many with keys
  static_assert(N % AH == 0 && NV >= AH, "the next step begins with the same register, and with values");
  // operand i: the first values (when they are read the keys may not have come yet), then all keys, then the other values
  auto value_of = [](int i) { return i < AH ? i : i < AH + NV ? -1 : i - NV; };
  auto read = [&](int i) {
    const int b = i < N ? block - 1 : block, k = i < N ? i : i - N, v = value_of(k);
    ahead.x[i % AH] = v >= 0 ? step_value<D>(ring, b, v / (D / 32), v % (D / 32)) : step_key<D, PAD>(ring, block + 1, k - AH, d);
  };
  const float base = R.m == -INFINITY ? 0.f : R.m;
  float p[8], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; ++i) next.x[i] = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const Piece y = ahead.x[i % AH];
    const int v = value_of(i);
    if (v >= 0)
      R.o[v % (D / 32)] = step_product(y, before.w[v / (D / 32)], R.o[v % (D / 32)]);
    else
      next.x = step_product(y, __builtin_bit_cast(bf16x8, R.q[i - AH]), next.x);
#pragma unroll
    for (int e = i * 16 / N; e < (i + 1) * 16 / N; ++e) {  // 16 probabilities over the N places
      p[e % 8] = step_exp(R, here, e, scale, base);
      if (e % 8 == 7) now.set(e / 8, p);
    }
    send(i);
    read(i + AH);
    if (i == N - 1) top = step_top(next);
    __builtin_amdgcn_sched_barrier(0);
  }
  return __any(top * scale > R.m + kWideSlack);
}

template <int D, bool PAD, bool SHARED>
__device__ __forceinline__ void step_item(const AttendArgs& a, const AttendCut& cut, const Partials& pt, int item, char* lds) {
  constexpr bool DRAFT = !SHARED;
  StepRing<D>& ring = *(StepRing<D>*)lds;
  Item it;
  if (!find_item<SHARED, true>(a, cut, item, pt, &it)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  // Of up to 64 rows two wavefronts have none: other ones in each of the two workgroups of a unit, which are mostly 256 apart.
  const int row0 = it.tile * kTile2 + 32 * ((wave + 2 * ((item >> 8) & 1)) & 3), r = row0 + (lane & 31);
  const Source src = source_of(a, it);
  int t0, t1;
  tiles_of<SHARED>(a, it, kTile2, &t0, &t1);
  const int key_first = t0 * kKeyTile, steps = (t1 - t0) * (kKeyTile / kStep);
  // (the first page numbers and the parents ahead of the queries and limits, which wait for loads of their own)
  int number = 0;
  Parents parents;
  if constexpr (DRAFT) parents.load(a, it.seg);
  if (steps > 0) number = src.table[min(key_first + (lane >> 1) * kStep + 16 * (lane & 1), src.last) >> src.shift];
  StepRows<D, DRAFT> rows;
  rows.odd = 0;
  rows.z = 0.f;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) rows.o[n][i] = 0.f;
  const int all = SHARED ? least_limit<true>(a, it.seg) : 0;
  const int context = DRAFT ? context_of(it.seg.len, it.seg.rows / a.G) : 0;
  const bool in = r < it.seg.rows;
  rows.lim = in ? row_limit<SHARED, true>(a, it.seg, r, all) : 0;
  rows.m = in ? -INFINITY : 0.f;                           // rows that are not there have logits 0: no reference to move for them
  {
    const int i = (int)((uint32_t)r / (uint32_t)a.G);
    const __bf16* q = (const __bf16*)a.q + (int64_t)(it.seg.c0 + i) * a.qt + (int64_t)(it.h * a.G + (r - i * a.G)) * a.qh;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) rows.q[c] = in && 16 * c + 8 * h < a.d ? *(const Piece*)(q + 16 * c + 8 * h) : Piece{0, 0, 0, 0};
  }
  StepWindow window = {};
  StepLane<D> at;
  if (steps > 0) window.start(src, key_first, number);     // (a row without tokens has no page number)
  at.template set<PAD>(src, wave);
  const uint32_t to_k = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&ring.k[0][wave >> 1][(wave & 1) * kStepLoads<D>][0];
  const uint32_t to_v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&ring.v[0][8 * wave][0];
  constexpr uint32_t kSlot = sizeof(ring.k[0]);            // (of a step's values too)
  static_assert(sizeof(ring.v[0]) == kSlot, "keys and values of a step take the same room");
  int64_t place = 0;                                       // of the step whose keys were sent last
  auto send_values = [&](int step, int64_t from) {
#pragma unroll
    for (int i = 0; i < kStepLoads<D>; ++i) send_to_lds(to_v + (uint32_t)(step & 3) * kSlot + i * 1024u, src.v + from, at.v[i]);
  };
  auto send_keys = [&](int step) {
    place = window.place(src, step, wave >> 1);
#pragma unroll
    for (int i = 0; i < kStepLoads<D>; ++i) send_to_lds(to_k + (uint32_t)(step & 3) * kSlot + i * 1024u, src.k + place, at.k[i]);
  };
  if (steps > 0) {                                         // (an item that is not empty has two steps at least)
    send_keys(0);
    send_values(0, place);
    send_keys(1);
    send_values(1, place);
    if (steps > 2) send_keys(2);
  }
  const uint32_t least = wave_min(in ? (uint32_t)(DRAFT ? context : rows.lim) : 0x7fffffffu), most = wave_max((uint32_t)rows.lim);
  if constexpr (DRAFT) {
    TreeLds<kTile2, true>& tree = *(TreeLds<kTile2, true>*)(lds + sizeof(StepRing<D>));
    rows.base = it.seg.len - it.seg.rows / a.G;
    rows.bits[0] = tree.bits[min((int)((uint32_t)r / (uint32_t)a.G) - (int)((uint32_t)(it.tile * kTile2) / (uint32_t)a.G), kTile2 - 1)];
    if (t1 * kKeyTile > context) read_tree<kTile2>(a, it.seg, parents, it.tile * kTile2, tree);      // (else no key of the draft is looked at)
  }
  const int all_see = SHARED ? all : context;              // keys that all rows of the workgroup see
  const float scale = a.scale * kLog2e;
  const int plain_end = min(steps, (all_see - key_first) / kStep);
  bool bad = false;
  int s = 0;
  // Step s begins: its values and the keys of s + 1 have landed, everybody's after the barrier, behind which nobody reads what step s - 1 was
  // the last to read: the places that step s sends to, V of s + 2 and K of s + 3.  Sent later than what is waited for: V of s + 1 and K of
  // s + 2, kStepLoads each.  Every step has one barrier, wherever a wavefront comes to it.
  auto begin = [&]() {
    if (s + 2 < steps) __builtin_amdgcn_s_waitcnt(0x0070 | (2 * kStepLoads<D>)); else __builtin_amdgcn_s_waitcnt(0x0070);   // and LDS reads
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();                          // (the fences of __syncthreads would wait for all sends)
    asm volatile("" ::: "memory");
  };
  auto send = [&]() {
    if (s + 2 < steps) send_values(s + 2, place);
    if (s + 3 < steps) send_keys(s + 3);
  };
  // The same one by one, beside products, which a wavefront would wait with while the four go out.
  struct Sends {
    const char* v;
    const char* k;
    uint32_t to_v, to_k, values, keys;
  };
  auto sends = [&]() {
    Sends x;
    x.values = s + 2 < steps ? 1u : 0u;
    x.keys = s + 3 < steps ? 1u : 0u;
    x.v = src.v + place;
    if (s + 3 < steps) place = window.place(src, s + 3, wave >> 1);
    x.k = src.k + place;
    x.to_v = to_v + (uint32_t)((s + 2) & 3) * kSlot;
    x.to_k = to_k + (uint32_t)((s + 3) & 3) * kSlot;
    return x;
  };
  auto send_one = [&](const Sends& x, int i) {
    constexpr int EVERY = D / 8 / (2 * kStepLoads<D>);     // products between two sends
    const int n = i / EVERY;
    if (i % EVERY != 0) return;
    if (n < kStepLoads<D>) send_to_lds_if(x.values, x.to_v + n * 1024u, x.v, at.v[n]);
    else send_to_lds_if(x.keys, x.to_k + (n - kStepLoads<D>) * 1024u, x.k, at.k[n - kStepLoads<D>]);
  };
  auto plain = [&]() { return s < plain_end && s < window.bad; };
  while (most == 0 && s < steps) {                         // a wavefront without rows only fetches
    begin();
    send();
    ++s;
  }
  // some row's reference has to move for these logits
  auto rises = [&](const StepLogits& l) { return __any(step_top(l) * scale > rows.m + kWideSlack); };
  bool begun = false;
  while (s < steps) {
    // (A first step that every row sees gives them their references by itself: shared prompts 46.9 us with a general one, 46.2 so.)
    if (s > 0 || !plain()) {
      if (!begun) begin();
      begun = false;
      send();
      const uint32_t ok = window.in_range(s);
      bad = bad || ok != 3u;
      const int key0 = key_first + s * kStep;
      if (key0 < (int)most) step_general<D, PAD>(rows, ring, s, key0, ok, (int)least, (int)most, a.d, scale);
      ++s;
      // steps that every row sees, as long as no reference has to move
      if (!plain()) continue;
    }
    StepLogits l[2];
    StepWeights w[2];
    begin();
    step_logits<D, PAD>(rows, ring, s, a.d, l[0]);
    if (s == 0) {                                          // (nothing stands on another reference yet)
      const float top = step_top(l[0]) * scale;
      rows.m = fmaxf(top, __shfl_xor(top, 32));
    }
    if (rises(l[0])) {
      begun = true;
      continue;
    }
    send();
    step_logits<D, PAD>(rows, ring, s + 1, a.d, l[1]);     // (behind the last step: of no use, from whatever is there)
    step_weights(rows, l[0], scale, w[0]);
    ++s;
    StepAhead ahead;
#pragma unroll
    for (int i = 0; i < StepAhead::N; ++i) ahead.x[i] = step_value<D>(ring, s - 1, i / (D / 32), i % (D / 32));
    bool stop = rises(l[1]);
    // logits of step s in `here`, the probabilities of the one before in `before`
    auto run = [&](const StepLogits& here, StepLogits& next, const StepWeights& before, StepWeights& now) {
      begin();
      if (stop) {
        begun = true;
        return false;
      }
      const Sends to = sends();
      ++s;
      stop = step_all<D, PAD>(rows, ring, s - 1, a.d, scale, here, next, before, now, ahead, [&](int i) { send_one(to, i); });
      return true;
    };
    for (;;) {
      if (!plain() || !run(l[1], l[0], w[0], w[1])) break;
      if (!plain() || !run(l[0], l[1], w[1], w[0])) {
        w[0] = w[1];
        break;
      }
    }
    step_values<D>(rows, ring, s - 1, w[0]);
  }
  if (bad && lane == 0) paged_fault(a.map);
  const float z = rows.z + __shfl_xor(rows.z, 32);
  if (!in) return;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v[4] = {rows.o[n][4 * j], rows.o[n][4 * j + 1], rows.o[n][4 * j + 2], rows.o[n][4 * j + 3]};
      write_row<__bf16, 4>(a, it, pt, D, r, 32 * n + 8 * j + 4 * h, v, rows.m, z);
    }
}

}  // namespace

}  // namespace asl
