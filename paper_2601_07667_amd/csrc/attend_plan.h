// How the work of an attention call is cut, and which kernels take it: arithmetic for device and host.
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
ASL_HD bool groups_pay(unsigned long long keys, int key_bytes) { return keys * (unsigned long long)key_bytes >= kMinSaved; }

// How a kind of segments is worked on: by split items of 16 rows, or tiles of 64 or 128 (0: there are none).
constexpr int kNone = 0, kSplit = 16, kTile1 = 64, kTile2 = 128;

// The longest sequences whose pieces (of 128 keys or more) are joined within the launch.
constexpr int kJoinKeys = 2048;

// The kind for `segments` segments of up to `rows` rows and `keys` keys.  A split item has all four wavefronts' loads on their way and
// needs no barrier, a tile reads its keys once for 64 or 128 rows: calls of little work are bound by latency and are split
// (32 query heads, 8 KV heads, d = 128; us, split and tiles: 32 rows 512 keys 11, 23; 128 rows 512 keys 11, 27; 64 rows 4096 keys 18,
// 25), others are not (8 sequences, 4096 keys: 32 rows 34, 36, 64 rows 50, 38; 32768 keys: 32 rows 225, 208, 64 rows 357, 214).
// Tiles of 64 rows up to 64 (8 sequences, 32768 keys, 64 rows 214 us, with tiles of 128 228).
constexpr double kSplitWork = 524288.;     // tiles of 16 rows x keys x KV heads
// Pieces of tiles: about 512 of own keys, two a compute unit (one chunk of 512 tokens over 4096 keys 63 us, with 384 74), 384 of
// shared ones, beside which there are others (shared prompt of 32768 keys 88 us, with 512 93.5); at least 8 key tiles each
// (shared drafts 36 us, with 4 47).
ASL_HD AttendCut cut_for(bool tiles, int64_t rows, int64_t keys, int64_t segments, int Hk, bool shared) {
  const double work = (double)((rows + 15) / 16) * (double)keys * (double)segments * Hk;
  if (tiles && rows > 16 && work >= kSplitWork) return AttendCut{rows > 64 ? kTile2 : kTile1, shared ? 384 : 512, 8, 0};
  return AttendCut{kSplit, 512, 2, 0};
}

// What the host decides about a call.
struct AttendRule {
  AttendCut own, shared;
  int64_t most;            // rows of a KV head that a sequence has at most
  bool groups;             // prefixes are read apart if the device finds that they save enough
  bool joined;             // pieces are joined within the launch
};

// tiles: the type and head size have tile items; room: rows of pieces in the workspace.
ASL_HD AttendRule rule_for(bool tiles, int64_t total_q, int G, int Hk, int n_seqs, int n_groups, int max_q_len, int max_kv_len,
                           int key_bytes, int64_t room) {
  AttendRule r;
  const int64_t rows = total_q * G;                        // of a KV head
  r.most = (int64_t)max_q_len * G < rows ? (int64_t)max_q_len * G : rows;
  r.own = cut_for(tiles, r.most, max_kv_len, n_seqs, Hk, false);
  r.shared = cut_for(tiles, n_groups > 0 ? rows / n_groups : 0, max_kv_len, n_groups, Hk, true);
  r.shared.cap = max_partials(r.shared, rows, Hk);
  // a sequence whose own rows fill a tile gains nothing, and groups cannot save more than all sequences' keys but one each (kMinSaved);
  // every row of a group is joined from two parts, for which there has to be room
  const double most_saved = (double)(n_seqs - n_groups) * (double)max_kv_len * (double)key_bytes;
  r.groups = n_groups > 0 && r.own.rows != kTile2 && most_saved >= (double)kMinSaved && r.shared.cap + rows * Hk <= room;
  if (!r.groups) r.shared.cap = 0;
  r.own.cap = room - r.shared.cap;
  // few pieces are joined by the workgroup that brings the last one
  r.joined = !r.groups && r.own.rows == kSplit && max_kv_len <= kJoinKeys;
  return r;
}

// Elements that one store to a row of `out` takes, of `held` neighbouring ones that a thread has: 16 bytes at most, since d and the strides
// of `out` are whole multiples of those and need not be of more (d = 100 in fp32: the thread that has elements 96 .. 103 stores four).
ASL_HD constexpr int store_elements(int held, int bytes) { return held * bytes > 16 ? 16 / bytes : held; }

}  // namespace asl
