// Reads commands from its input and prints what the library's rules for the paged calls come to (built and run by tests/test_paged_rules.py).
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
    if (!std::strcmp(what, "stores")) {
      // bytes of an element, elements that a thread holds, padded and true head size: whether the threads' stores to a row take each
      // of its elements once and nothing behind it
      const int bytes = (int)num(), held = (int)num(), D = (int)num(), d = (int)num(), w = asl::store_elements(held, bytes);
      std::vector<int> hit(D + 64);
      for (int e0 = 0; e0 < D; e0 += held)
        for (int x0 = 0; x0 < held; x0 += w)
          for (int x = 0; x < w && e0 + x0 < d; ++x) ++hit[e0 + x0 + x];
      bool ok = held % w == 0;
      for (int e = 0; e < D + 64; ++e) ok = ok && hit[e] == (e < d ? 1 : 0);
      std::printf("%d %d\n", ok ? 1 : 0, w);
    } else if (!std::strcmp(what, "rule")) {
      // whether there are tiles, query tokens, G, Hk, sequences, groups, most queries and keys, bytes of a key, room; then the groups'
      // shared keys: kinds of own and shared segments, whether the host leaves groups on, whether the device does, joined in the launch
      const bool tiles = num() != 0;
      const long long total = num();
      const int G = (int)num(), Hk = (int)num(), seqs = (int)num(), groups = (int)num(), mq = (int)num(), mk = (int)num(), bytes = (int)num();
      const long long room = num(), keys = num();
      const asl::AttendRule r = asl::rule_for(tiles, total, G, Hk, seqs, groups, mq, mk, bytes, room);
      std::printf("%d %d %d %d %d\n", r.own.rows, r.shared.rows, r.groups ? 1 : 0, asl::groups_pay((unsigned long long)keys, bytes) ? 1 : 0,
                  r.joined ? 1 : 0);
    } else if (!std::strcmp(what, "room")) {
      // n limits (query rows, head size) in turn: the room after each
      asl::PagedRoom r = {0, 0};
      for (int n = (int)num(); n > 0; --n) {
        const int rows = (int)num(), dim = (int)num();
        r = asl::room_for(r, rows, dim);
        std::printf("%d %d\n", r.rows, r.dim);
      }
    } else if (!std::strcmp(what, "kept")) {
      std::printf("%d\n", asl::kPagedKept);
    }
  }
  return 0;
}
