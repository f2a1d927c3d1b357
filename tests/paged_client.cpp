// Reads commands from its input and prints what the library's own headers make of them (built and run by tests/test_paged.py):
//   pages, rows, attn + their fields: status and message of the check;  index: tables of numbers, in and out of range.
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "attend_plan.h"
#include "paged_check.h"

static long long num() {
  long long x = 0;
  if (std::scanf("%lld", &x) != 1) x = 0;
  return x;
}

static asl_pages read_pages() {
  asl_pages p;
  p.n_q_heads = (int)num(); p.n_kv_heads = (int)num(); p.head_dim = (int)num(); p.dtype = (int)num();
  p.page_size = (int)num(); p.n_pages = (int)num(); p.n_rows = (int)num(); p.row_stride = (int)num();
  p.stride_page = num(); p.stride_head = num(); p.stride_tok = num();
  p.scale = 0.f;
  p.flags = (int)num();
  return p;
}

int main() {
  char what[16];
  while (std::scanf("%15s", what) == 1) {
    const char* why = "";
    if (!std::strcmp(what, "pages")) {
      const asl_pages p = read_pages();
      const int st = asl::pages_status(&p, &why);
      std::printf("%d %s\n", st, why);
    } else if (!std::strcmp(what, "rows")) {
      const asl_pages p = read_pages();
      asl_rows r;
      r.n_src = (int)num(); r.idx_rows = 1;
      r.k_stride_head = num(); r.k_stride_tok = num(); r.v_stride_head = num(); r.v_stride_tok = num();
      const int st = asl::rows_status(p, &r, &why);
      std::printf("%d %s\n", st, why);
    } else if (!std::strcmp(what, "attn")) {
      const asl_pages p = read_pages();
      asl_attn a;
      a.n_seqs = (int)num(); a.total_q = (int)num(); a.max_q_len = (int)num(); a.max_kv_len = (int)num();
      a.n_groups = (int)num(); a.flags = (int)num();
      a.q_stride_tok = num(); a.q_stride_head = num(); a.out_stride_tok = num(); a.out_stride_head = num();
      const int st = asl::attn_status(p, &a, &why);
      std::printf("%d %s\n", st, why);
    } else if (!std::strcmp(what, "null")) {
      const asl_pages p = {};
      std::printf("%d %d %d\n", asl::pages_status(nullptr, &why), asl::rows_status(p, nullptr, &why), asl::attn_status(p, nullptr, &why));
    } else if (!std::strcmp(what, "index")) {
      // n_pages n_rows row_stride ps, the table's entries, the lengths, then row and position: length's verdict and the offset
      asl_pages p = {};
      p.n_q_heads = p.n_kv_heads = 1; p.head_dim = 8;
      p.n_pages = (int)num(); p.n_rows = (int)num(); p.row_stride = (int)num(); p.page_size = (int)num();
      p.stride_tok = 8; p.stride_head = 8LL * p.page_size; p.stride_page = p.stride_head;
      std::vector<int32_t> table((size_t)p.n_rows * p.row_stride), len(p.n_rows);
      for (int32_t& x : table) x = (int32_t)num();
      for (int32_t& x : len) x = (int32_t)num();
      const asl::PageMap m = asl::page_map(p, 2, table.data(), len.data(), nullptr);
      const int r = (int)num(), pos = (int)num();
      int L = -7;
      const bool ok = asl::row_length(m, r, &L);
      std::printf("%d %d %lld\n", ok ? 1 : 0, L, (long long)asl::token_offset(m, r, pos));
    } else if (!std::strcmp(what, "cut")) {
      // rows of a tile, target, least tiles, KV heads, the segments' rows and spans: whether every share is whole, the items and partial
      // rows that the cut gives and the most that a launch makes room for
      asl::AttendCut c = {};
      c.rows = (int)num(); c.target = (int)num(); c.min_tiles = (int)num();
      const int Hk = (int)num(), n = (int)num();
      std::vector<long long> rows(n), span(n);
      unsigned long long work = 0;
      long long all_rows = 0;
      for (int i = 0; i < n; ++i) {
        rows[i] = num();
        span[i] = num();
        all_rows += rows[i];
        work += (unsigned long long)((rows[i] + c.rows - 1) / c.rows) * Hk * (span[i] < 1 ? 1 : span[i]);
      }
      const long long per = asl::tiles_per_item(c, work);
      long long items = 0, partial = 0;
      bool ok = true;
      for (int i = 0; i < n; ++i) {
        const int k = asl::splits_of((int)span[i], per);
        items += (rows[i] + c.rows - 1) / c.rows * Hk * k;
        partial += rows[i] * Hk * k;
        int at = 0;
        for (int s = 0; s < k; ++s) {
          int t0, t1;
          asl::split_range((int)span[i], k, s, &t0, &t1);
          ok = ok && t0 == at && t1 >= t0 && t1 - t0 <= per;
          at = t1;
        }
        ok = ok && at == span[i];
      }
      std::printf("%d %lld %lld %lld %lld\n", ok ? 1 : 0, items, (long long)asl::max_items(c, all_rows, n, Hk), partial,
                  (long long)asl::max_partials(c, all_rows, Hk));
    } else if (!std::strcmp(what, "shared")) {
      const int stated = (int)num(), first = (int)num(), members = (int)num();
      std::printf("%d\n", asl::shared_tokens(stated, first, members));
    } else if (!std::strcmp(what, "seq")) {
      const int n = (int)num();
      std::vector<int32_t> cu(n + 1);
      for (int32_t& x : cu) x = (int32_t)num();
      const int j = (int)num();
      std::printf("%d\n", asl::sequence_of(cu.data(), n, j));
    }
  }
  return 0;
}
