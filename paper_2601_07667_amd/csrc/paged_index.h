// Index arithmetic of the paged cache, for device and host.  A page holds `ps` tokens of every KV head; a sequence is a row of
// `table` (page numbers, in order) and a length in `kv_len`.  Table, lengths and counts are the caller's device memory, so the
// host knows none of them: every number that a kernel reads from there and uses as an index is checked against the limits here
// first, and what is out of range is left out and raises the fault word.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define ASL_HD __host__ __device__ __forceinline__
#else
#define ASL_HD inline
#endif

namespace asl {

constexpr uint32_t kFaultPaged = 2;        // bit of the fault word: a row, length, token or page number out of range
constexpr int kPagedMaxSeqs = 4096;        // sequences of one call
constexpr int kMaxFresh = 65536;           // pages that one call takes
constexpr int kCutRows = 131072;           // rows of partial results beside one for each row's own and shared keys
constexpr int kPagedMaxDim = 256;          // head_dim of asl_paged_attention
constexpr int kTreeNodes = 512;            // nodes of a draft (asl_tree_attention, asl_pages_accept)
constexpr int kPlanNodes = 16384;          // nodes of a draft (asl_pages_plan): a node's depth is a walk of as many loads that depend on each other
constexpr int kTreeWords = kTreeNodes / 32;
constexpr int kPagedRowsHeld = 131072;     // query rows beyond which the workspace does not grow
constexpr int kPagedKept = 7;              // workspaces that a context outgrows at most (see room_for)

struct PageMap {
  const int32_t* table;                    // [n_rows][row_stride]
  const int32_t* kv_len;                   // [n_rows]
  uint32_t* fault;
  int32_t n_pages, n_rows, row_stride;
  int32_t ps, ps_shift;                    // tokens of a page, a power of two
  int64_t page, head, tok;                 // strides of the pages in bytes
};

// Index i with cu[i] <= j < cu[i + 1] of an ascending cu[0..n]; whatever cu holds, one from 0 to n - 1.
ASL_HD int sequence_of(const int32_t* cu, int n, int j) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= j) lo = mid; else hi = mid;
  }
  return lo;
}

// Whether row r and its length are in range; *len gets the length, 0 if they are not.
ASL_HD bool row_length(const PageMap& m, int r, int* len) {
  *len = 0;
  if ((uint32_t)r >= (uint32_t)m.n_rows) return false;
  const int L = m.kv_len[r];
  if (L < 0 || L > (int64_t)m.row_stride * m.ps) return false;
  *len = L;
  return true;
}

// Byte offset of token `pos` of row r in the pages of KV head 0, or -1 if row, position or page number are out of range.
ASL_HD int64_t token_offset(const PageMap& m, int r, int pos) {
  if ((uint32_t)r >= (uint32_t)m.n_rows || pos < 0 || (pos >> m.ps_shift) >= m.row_stride) return -1;
  const int page = m.table[(int64_t)r * m.row_stride + (pos >> m.ps_shift)];
  if ((uint32_t)page >= (uint32_t)m.n_pages) return -1;
  return (int64_t)page * m.page + (int64_t)(pos & (m.ps - 1)) * m.tok;
}

}  // namespace asl
