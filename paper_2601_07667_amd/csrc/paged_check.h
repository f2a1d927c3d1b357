// The paged calls' checks of the structs that they are given, and the size of their workspace.  Host code, without a GPU.
#pragma once
#include <stdint.h>

#include "asl.h"
#include "paged_index.h"

namespace asl {

inline int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

inline int bytes_of(int dtype) { return dtype == ASL_BF16 ? 2 : 4; }

// What a workspace of the paged calls has room for.
struct PagedRoom {
  int32_t rows;            // query rows (as far as the pieces of their results grow with them)
  int32_t dim;             // padded head size
};

// The room that limits need beside what there is: never less in either measure, rows a power of two.  So a context's limits may go up and
// down in any order, and of 6 sizes by 3 it takes at most 7 steps from the first workspace to the largest.
inline PagedRoom room_for(const PagedRoom& have, int32_t max_query_rows, int32_t max_head_dim) {
  PagedRoom r = {4096, max_head_dim <= 64 ? 64 : max_head_dim <= 128 ? 128 : 256};
  while (r.rows < max_query_rows && r.rows < kPagedRowsHeld) r.rows *= 2;
  if (r.rows < have.rows) r.rows = have.rows;
  if (r.dim < have.dim) r.dim = have.dim;
  return r;
}

// Strides and rows that 16-byte pieces take.
inline bool whole_pieces(int64_t elements, int dtype) { return elements * bytes_of(dtype) % 16 == 0; }

// ASL_OK, or what is wrong with p and *why.
inline asl_status pages_status(const asl_pages* p, const char** why) {
  auto no = [&](asl_status st, const char* text) { *why = text; return st; };
  if (!p) return no(ASL_EINVAL, "pages is null");
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0)
    return no(ASL_EINVAL, "need Hq >= 1, Hk >= 1, Hq % Hk == 0");
  if (p->head_dim < 1) return no(ASL_EINVAL, "head_dim must be >= 1");
  if (p->page_size < 1 || p->n_pages < 1 || p->n_rows < 1 || p->row_stride < 1)
    return no(ASL_EINVAL, "page_size, n_pages, n_rows and row_stride must be >= 1");
  if (p->flags != 0) return no(ASL_EINVAL, "unknown bits in flags");
  if (p->dtype != ASL_BF16 && p->dtype != ASL_F32) return no(ASL_EUNSUPPORTED, "dtype not supported");
  if (p->page_size < 16 || p->page_size > 4096 || (p->page_size & (p->page_size - 1)) != 0)
    return no(ASL_EUNSUPPORTED, "page_size must be a power of two from 16 to 4096");
  if ((int64_t)p->row_stride * p->page_size > (int64_t(1) << 30))
    return no(ASL_EUNSUPPORTED, "a table row of more than 2^30 tokens");
  if (p->n_q_heads > 65535) return no(ASL_EUNSUPPORTED, "more than 65535 heads");
  if (p->head_dim > 65536) return no(ASL_EUNSUPPORTED, "head_dim > 65536");
  if (p->stride_tok < p->head_dim || p->stride_head < 0 || p->stride_page < 0)
    return no(ASL_EINVAL, "page strides must satisfy stride_tok >= d, stride_head >= 0, stride_page >= 0");
  if (!whole_pieces(p->head_dim, p->dtype) || !whole_pieces(p->stride_tok, p->dtype) ||
      !whole_pieces(p->stride_head, p->dtype) || !whole_pieces(p->stride_page, p->dtype))
    return no(ASL_EUNSUPPORTED, "rows and strides of pages must be multiples of 16 bytes");
  if (p->stride_tok > (int64_t(1) << 24)) return no(ASL_EUNSUPPORTED, "a token stride of more than 2^24 elements");
  return ASL_OK;
}

inline asl_status rows_status(const asl_pages& p, const asl_rows* r, const char** why) {
  auto no = [&](asl_status st, const char* text) { *why = text; return st; };
  if (!r) return no(ASL_EINVAL, "src is null");
  if (r->n_src < 0) return no(ASL_EINVAL, "n_src must be >= 0");
  if (r->k_stride_tok < p.head_dim || r->v_stride_tok < p.head_dim || r->k_stride_head < 0 || r->v_stride_head < 0)
    return no(ASL_EINVAL, "source strides must satisfy stride_tok >= d, stride_head >= 0");
  if (!whole_pieces(r->k_stride_tok, p.dtype) || !whole_pieces(r->k_stride_head, p.dtype) ||
      !whole_pieces(r->v_stride_tok, p.dtype) || !whole_pieces(r->v_stride_head, p.dtype))
    return no(ASL_EUNSUPPORTED, "strides of k and v must be multiples of 16 bytes");
  return ASL_OK;
}

inline asl_status attn_status(const asl_pages& p, const asl_attn* a, const char** why) {
  auto no = [&](asl_status st, const char* text) { *why = text; return st; };
  if (!a) return no(ASL_EINVAL, "attn is null");
  if (a->n_seqs < 0 || a->total_q < 0 || a->max_q_len < 0 || a->max_kv_len < 0 || a->n_groups < 0)
    return no(ASL_EINVAL, "n_seqs, total_q, max_q_len, max_kv_len and n_groups must be >= 0");
  if (a->n_groups > a->n_seqs) return no(ASL_EINVAL, "more groups than sequences");
  if (a->flags & ~ASL_ATTN_CAUSAL) return no(ASL_EINVAL, "unknown bits in flags");
  if (a->q_stride_tok < 0 || a->q_stride_head < 0 || a->out_stride_tok < 0 || a->out_stride_head < 0)
    return no(ASL_EINVAL, "strides of q and out must be >= 0");
  if (!whole_pieces(a->q_stride_tok, p.dtype) || !whole_pieces(a->q_stride_head, p.dtype) ||
      !whole_pieces(a->out_stride_tok, p.dtype) || !whole_pieces(a->out_stride_head, p.dtype))
    return no(ASL_EUNSUPPORTED, "strides of q and out must be multiples of 16 bytes");
  return ASL_OK;
}

inline PageMap page_map(const asl_pages& p, int eb, const int32_t* table, const int32_t* kv_len, uint32_t* fault) {
  PageMap m;
  m.table = table;
  m.kv_len = kv_len;
  m.fault = fault;
  m.n_pages = p.n_pages;
  m.n_rows = p.n_rows;
  m.row_stride = p.row_stride;
  m.ps = p.page_size;
  m.ps_shift = log2_of(p.page_size);
  m.page = p.stride_page * eb;
  m.head = p.stride_head * eb;
  m.tok = p.stride_tok * eb;
  return m;
}

}  // namespace asl
