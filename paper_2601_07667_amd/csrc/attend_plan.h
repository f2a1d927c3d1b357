// How the work of an attention call is cut: index arithmetic for device and host.
//
// The queries of a sequence that share a KV head are its rows (token-major: row = token * G + head of the group), the keys that only
// it sees its span, in tiles of kKeyTile.  A group with a shared prefix has a second such segment: the rows of all its sequences over
// the prefix.  Work items are (segment, split of the span, tile of rows, KV head), one workgroup each.  Lengths are known on the
// device alone, so a launch has as many workgroups as the cut can give at most (max_items), and each finds its own item.
#pragma once
#include <stdint.h>

#include "paged_index.h"

namespace asl {

constexpr int kKeyTile = 64;

struct AttendCut {
  int32_t rows;            // rows of a tile (M)
  int32_t target;          // items that the spans are cut into, about
  int32_t min_tiles;       // key tiles of an item, at least (but for a segment's last)
  int64_t cap;             // rows of partial results that there is room for
};

// Key tiles of an item: as many as give about `target` items of `work` (row tiles x heads x key tiles).
ASL_HD int64_t tiles_per_item(const AttendCut& c, unsigned long long work) {
  const int64_t t = (int64_t)((work + (unsigned long long)c.target - 1) / (unsigned long long)c.target);
  return t > c.min_tiles ? t : c.min_tiles;
}

ASL_HD int splits_of(int span, int64_t per_item) { return span < 1 ? 1 : (int)((span + per_item - 1) / per_item); }

// Tiles [*t0, *t1) of `span` that split s of n takes; equal shares, the first ones a tile longer.
ASL_HD void split_range(int span, int n, int s, int* t0, int* t1) {
  const int each = span / n, more = span - each * n;
  *t0 = s * each + (s < more ? s : more);
  *t1 = *t0 + each + (s < more ? 1 : 0);
}

// Items that a launch over `segments` segments with `rows` rows of one KV head in all can have at most: each segment has
// ceil(rows / M) row tiles, each cut into ceil(span / per_item) pieces.
ASL_HD int64_t max_items(const AttendCut& c, int64_t rows, int64_t segments, int Hk) {
  return c.target + Hk * (rows / c.rows + segments);
}

// Rows of partial results that such a launch can leave at most.
ASL_HD int64_t max_partials(const AttendCut& c, int64_t rows, int Hk) { return rows * Hk + (int64_t)c.target * c.rows; }

// Tokens of a group that a segment of its own takes: whole key tiles of what is stated and there; none for a group of one.
constexpr int kMinShared = 128;
ASL_HD int shared_tokens(int stated, int first_len, int members) {
  if (members < 2) return 0;
  const int p = (stated < first_len ? stated : first_len) & ~(kKeyTile - 1);
  return p < kMinShared ? 0 : p;
}

// Bytes of K and V that a call's groups have to save for their prefixes to be read apart; read by each sequence they come from the
// caches, and nothing has to be joined (d = 128; us, apart and by each: 32 query heads, 8 KV heads, one group of 64, prefix 512
// (132 MB) 29, 20, 1024 (264 MB) 30, 29, 2090 32, 74; 8 groups of 6, 1024 (168 MB) 37, 39; 28 heads, 4 KV heads, 8 groups of 6,
// 1024 (84 MB) 34, 27, 2090 (171 MB) 37, 45).
constexpr unsigned long long kMinSaved = 128ull << 20;

// Elements that one store to a row of `out` takes, of `held` neighbouring ones that a thread has: 16 bytes at most, since d and the strides
// of `out` are whole multiples of those and need not be of more (d = 100 in fp32: the thread that has elements 96 .. 103 stores four).
ASL_HD constexpr int store_elements(int held, int bytes) { return held * bytes > 16 ? 16 / bytes : held; }

}  // namespace asl
