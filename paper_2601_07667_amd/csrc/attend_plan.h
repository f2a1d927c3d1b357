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

// (Divisions of 64 bits take a wavefront about 1000 cycles each, and every one works the cut out: of 32 bits where the numbers allow it.)
// Key tiles of an item: as many as give about `target` items of `work` (row tiles x heads x key tiles).
ASL_HD int64_t tiles_per_item(const AttendCut& c, unsigned long long work) {
  const unsigned long long up = work + (unsigned long long)c.target - 1;
  const int64_t t = up >> 32 == 0 ? (int64_t)((uint32_t)up / (uint32_t)c.target) : (int64_t)(up / (unsigned long long)c.target);
  return t > c.min_tiles ? t : c.min_tiles;
}

ASL_HD int splits_of(int span, int64_t per_item) {
  return per_item >= span ? 1 : (int)(((uint32_t)span - 1u) / (uint32_t)per_item) + 1;   // (spans are below 2^31, and so then is per_item)
}

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

// Row tile and split of item e of a tree's segment, whose head is e % Hk, for Hk < 8.  Items of the same keys are to be a multiple of 8 apart,
// so that one die's L2 has the keys for all their row tiles: as many splits take turns as make a multiple of 8 with the heads.  (Not in the
// last turns where those are fewer.)  60 nodes of 7 heads a group behind 131089 keys, us, with the row tiles in turn and so: 4 heads 193, 187;
// with 3 splits in turn for 3 heads, 2 for 5 to 7, and so: 3 heads 141, 126; 5 300, 261; 6 307, 303; 7 402, 342.
ASL_HD void tree_turn(uint32_t e, uint32_t Hk, uint32_t tiles, uint32_t splits, uint32_t* tile, uint32_t* split) {
  const uint32_t by = Hk % 4 == 0 ? 2u : Hk % 2 == 0 ? 4u : 8u, block = Hk * tiles * by;
  const uint32_t k = e / block, at = (e - k * block) / Hk, left = splits - k * by, n = by < left ? by : left;
  *tile = tiles - 1u - at / n;
  *split = k * by + at % n;
}

// Items of a launch: 256 threads each.  One of 2^32 threads or more in x does not fail: it runs with their number modulo 2^32.
constexpr int64_t kMostItems = (int64_t(1) << 32) / 256;

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

// The same for drafted trees, which have tiles of 128 rows alone (attend_steps.h).  An item takes 10 us to begin and its pieces 9 to 16 to be
// joined, so where there are tiles for three quarters of the units a span of up to 128 key tiles is one piece (32 sequences of 2300
// keys, 16 to 32 nodes, 8 heads: 82 us, in two pieces each 108).  Where by the caller's word no sequence is longer than that, every span is
// one (one item in all is wanted), however many keys it turns out to have, and no launch looks for pieces to join (83 us, 80 so).  The tiles are
// counted as if every draft had as many nodes as the caller states for the longest: few and uneven ones are not cut either, and take longer
// (drafts of 200, 8, 8 and 8 nodes on 8192 keys, 4 heads a group, 8 heads: 180 us, apart 76 and 39).  Where there
// are fewer tiles, spans are cut for two items a unit (60 nodes on 131089 keys, 4 heads: 186 us, with 384 items 196, with 256 207).  Shared
// ones into about 192 (8 prompts of 2090 keys for 6 sequences each: 46.6 us, with 128 46.8, with 256 47.5, with 384 54.5, with 96 64).
ASL_HD AttendCut cut_for_tree(bool tiles, int64_t rows, int64_t keys, int64_t segments, int Hk, bool shared) {
  AttendCut c = cut_for(tiles, rows, keys, segments, Hk, shared);
  if (c.rows == kSplit) return c;
  const int64_t row_tiles = (rows + kTile2 - 1) / kTile2 * segments * Hk;
  if (!shared && row_tiles >= 192 && keys <= 128 * kKeyTile) return AttendCut{kTile2, 1, 128, 0};
  return AttendCut{kTile2, shared ? 192 : 512, !shared && row_tiles >= 192 ? 128 : 8, 0};
}

// What the host decides about a call.
struct AttendRule {
  AttendCut own, shared;
  int64_t most;            // rows of a KV head that a sequence has at most
  bool groups;             // prefixes are read apart if the device finds that they save enough
  bool joined;             // pieces are joined within the launch
  bool single;             // there are none to join
};

// tiles: the type and head size have tile items; room: rows of pieces in the workspace.
ASL_HD AttendRule rule_for(bool tiles, int64_t total_q, int G, int Hk, int n_seqs, int n_groups, int max_q_len, int max_kv_len,
                           int key_bytes, int64_t room, bool tree = false) {
  AttendRule r;
  const int64_t rows = total_q * G;                        // of a KV head
  r.most = (int64_t)max_q_len * G < rows ? (int64_t)max_q_len * G : rows;
  r.own = (tree ? cut_for_tree : cut_for)(tiles, r.most, max_kv_len, n_seqs, Hk, false);
  r.shared = (tree ? cut_for_tree : cut_for)(tiles, n_groups > 0 ? rows / n_groups : 0, max_kv_len, n_groups, Hk, true);
  r.shared.cap = max_partials(r.shared, rows, Hk);
  // a sequence whose own rows fill a tile reads its keys once for all of them; groups cannot save more than all sequences' keys but one each
  // (kMinSaved).  Drafts share up to one tile of rows, a bound that was not measured out: just above it sharing would pay (64 sequences behind
  // 33024 keys, 4 heads a group: 32 nodes 1183 us, 33 nodes, each reading the prefix for two tiles of rows, 1846).  And every row of a group is joined from two parts, for which there has to be room
  const double most_saved = (double)(n_seqs - n_groups) * (double)max_kv_len * (double)key_bytes;
  r.groups = n_groups > 0 && (tree ? r.most <= kTile2 : r.own.rows != kTile2) && most_saved >= (double)kMinSaved && r.shared.cap + rows * Hk <= room;
  if (!r.groups) r.shared.cap = 0;
  r.own.cap = room - r.shared.cap;
  // few pieces are joined by the workgroup that brings the last one
  r.joined = !r.groups && r.own.rows == kSplit && max_kv_len <= kJoinKeys;
  r.single = !r.groups && r.own.target == 1;
  return r;
}

// Elements that one store to a row of `out` takes, of `held` neighbouring ones that a thread has: 16 bytes at most, since d and the strides
// of `out` are whole multiples of those and need not be of more (d = 100 in fp32: the thread that has elements 96 .. 103 stores four).
ASL_HD constexpr int store_elements(int held, int bytes) { return held * bytes > 16 ? 16 / bytes : held; }

}  // namespace asl
