// Reads commands from its input and prints what the library's rules for the drafting calls come to (built and run by tests/test_draft.py).
#include <cstdio>
#include <cstring>
#include <vector>

#include "attend_plan.h"
#include "paged_check.h"

static long long num() {
  long long x = 0;
  if (std::scanf("%lld", &x) != 1) x = 0;
  return x;
}

int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    const char* why = "";
    if (!std::strcmp(what, "rotation")) {
      asl_rotation r;
      r.n_q_heads = (int)num(); r.n_kv_heads = (int)num(); r.head_dim = (int)num(); r.dtype = (int)num(); r.rot_dim = (int)num();
      r.pairs = (int)num(); r.flags = (int)num();
      r.magnitude = 0.f;
      int64_t* s = &r.q_stride_tok;
      for (int i = 0; i < 10; ++i) s[i] = num();
      const int st = asl::rotation_status(&r, &why);
      std::printf("%d %s\n", st, why);
    } else if (!std::strcmp(what, "width")) {
      // dtype, d, rot, pairs, alignment: bytes of a piece, and whether pieces of that size, as the kernel numbers them, take every element of
      // a head once and every pair's elements together
      asl_rotation r = {};
      r.dtype = (int)num(); r.head_dim = (int)num(); r.rot_dim = (int)num(); r.pairs = (int)num();
      const long long align = num();
      const int W = asl::rotate_width(r, align), eb = asl::bytes_of(r.dtype), E = W / eb;
      const bool halves = r.pairs == ASL_PAIRS_HALVES;
      const int turned = halves ? r.rot_dim / 2 / E : r.rot_dim / E, units = turned + (r.head_dim - r.rot_dim) / E;
      std::vector<int> hit(r.head_dim + 64), copied(r.head_dim + 64);
      auto mark = [&](std::vector<int>& v, int byte) {
        for (int e = 0; e < E; ++e) ++v[byte / eb + e];
      };
      bool ok = W % eb == 0 && E >= 1 && (halves || E % 2 == 0) && align % (W == 16 ? 16 : eb) == 0;
      for (int u = 0; u < units; ++u) {
        mark(hit, !halves || u < turned ? u * W : r.rot_dim * eb + (u - turned) * W);
        if (halves && u < turned) mark(hit, r.rot_dim / 2 * eb + u * W);
        mark(copied, u * W);
        if (halves && (u + units) * W < r.head_dim * eb) mark(copied, (u + units) * W);
      }
      for (int e = 0; e < r.head_dim + 64; ++e) ok = ok && hit[e] == (e < r.head_dim ? 1 : 0) && copied[e] == (e < r.head_dim ? 1 : 0);
      std::printf("%d %d\n", ok ? 1 : 0, W);
    } else if (!std::strcmp(what, "tree")) {
      asl_attn a = {};
      a.flags = (int)num(); a.max_q_len = (int)num();
      const int st = asl::tree_status(a, &why);
      std::printf("%d %s\n", st, why);
    } else if (!std::strcmp(what, "rule")) {
      // total_q, G, Hk, sequences, groups, nodes of a draft, keys, bytes of a key: kinds of items, and the most pieces that are asked for
      long long x[8];
      for (long long& y : x) y = num();
      const asl::AttendRule r = asl::rule_for(true, x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], (int)x[5], (int)x[6], (int)x[7],
                                              1 << 20, true);
      std::printf("%d %d %d %d %d %d\n", r.own.rows, r.groups ? r.shared.rows : 0, (int)r.joined, (int)r.single, r.own.cap + r.shared.cap <= (1 << 20),
                  r.own.cap >= 0 && r.shared.cap >= 0);
    } else if (!std::strcmp(what, "null")) {
      asl_freqs f = {};
      double x;
      std::printf("%d %d %d\n", asl::rotation_status(nullptr, &why), asl::rotation_freqs(nullptr, &x), asl::rotation_freqs(&f, nullptr));
    }
  }
  return 0;
}
