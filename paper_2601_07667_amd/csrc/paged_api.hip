// The entry points of the paged cache: the workspace, the checks of arguments, the launches.
#include "context.h"
#include "paged_check.h"

namespace {

// The checks of asl_pages (paged_check.h), and the map that the kernels take.
asl_status check_pages(asl_ctx* ctx, const asl_pages* p, const int32_t* table, const int32_t* kv_len, asl::PageMap* m) {
  if (!ctx) return ASL_EINVAL;
  const char* why = "";
  const asl_status st = asl::pages_status(p, &why);
  if (st != ASL_OK) return fail(ctx, st, "%s", why);
  if (!ctx->paged.base) return fail(ctx, ASL_ENOMEM, "call asl_paged_reserve first");
  if (!table || !kv_len) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  *m = asl::page_map(*p, elem_bytes(p->dtype), table, kv_len, ctx->paged.fault);
  return ASL_OK;
}

asl_status check_count(asl_ctx* ctx, int32_t n) {
  if (n < 0) return fail(ctx, ASL_EINVAL, "the number of sequences must be >= 0");
  if (n > ctx->paged.max_seqs)
    return fail(ctx, ASL_ENOMEM, "%d sequences exceed the %d that asl_paged_reserve was called for", n, ctx->paged.max_seqs);
  return ASL_OK;
}

void set_row_pieces(int64_t row_bytes, int32_t* cpr, int32_t* shift) {
  *cpr = (int32_t)(row_bytes / 16);
  *shift = (*cpr & (*cpr - 1)) == 0 ? asl::log2_of(*cpr) : -1;
}

// Rows of pieces of attention's results: every row twice (its own and its shared keys; not for the largest calls, which have no need to
// share), and the pieces that long spans are cut into.
int64_t part_rows(int32_t query_rows) {
  return 2 * (int64_t)(query_rows < asl::kPagedRowsHeld ? query_rows : asl::kPagedRowsHeld) + asl::kCutRows;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

asl_status asl_paged_reserve(asl_ctx* ctx, int32_t max_seqs, int32_t max_query_rows, int32_t max_head_dim) {
  if (!ctx) return ASL_EINVAL;
  if (max_seqs < 1 || max_query_rows < 1 || max_head_dim < 1) return fail(ctx, ASL_EINVAL, "limits must be >= 1");
  if (max_seqs > asl::kPagedMaxSeqs) return fail(ctx, ASL_EUNSUPPORTED, "more than %d sequences per call", asl::kPagedMaxSeqs);
  if (max_head_dim > asl::kPagedMaxDim) return fail(ctx, ASL_EUNSUPPORTED, "head_dim > %d not supported", asl::kPagedMaxDim);
  asl::PagedWorkspace& ws = ctx->paged;
  const asl::PagedRoom room = asl::room_for({ws.room_rows, ws.room_dim}, max_query_rows, max_head_dim);
  if (!ws.base || room.rows != ws.room_rows || room.dim != ws.room_dim) {
    DeviceGuard guard(ctx->device);
    if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
    asl::PagedWorkspace w = {};
    size_t off = 0;
    auto take = [&](size_t bytes) {
      const size_t at = off;
      off += align_up(bytes);
      return at;
    };
    const size_t rows = (size_t)part_rows(room.rows);
    const size_t fault = take(sizeof(uint32_t)), forks = take((size_t)asl::kPagedMaxSeqs * sizeof(int4)),
                 fresh = take((size_t)asl::kMaxFresh * sizeof(int32_t)),
                 plan = take((size_t)2 * asl::kPagedMaxSeqs * sizeof(int4)),
                 group = take((size_t)asl::kPagedMaxSeqs * sizeof(int32_t)),
                 cut = take(sizeof(int32_t));
    const size_t part = take(rows * room.dim * sizeof(float)), part_mz = take(rows * sizeof(float2)),
                 arrived = take(rows * sizeof(uint32_t));
    char* base = nullptr;
    hipError_t e = hipMalloc(&base, off);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return fail(ctx, e == hipErrorOutOfMemory ? ASL_ENOMEM : ASL_EHIP, "workspace of %zu bytes: %s", off, hipGetErrorString(e));
    }
    e = hipMemset(base, 0, off);
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);  // calls may follow on any stream
    if (e != hipSuccess) {
      (void)hipFree(base);
      return hip_fail(ctx, e, "workspace");
    }
    w.base = base;
    w.room_rows = room.rows;
    w.room_dim = room.dim;
    w.fault = ws.base ? ws.fault : (uint32_t*)(base + fault);
    w.forks = (int4*)(base + forks);
    w.fresh = (int32_t*)(base + fresh);
    w.plan = (int4*)(base + plan);
    w.group = (int32_t*)(base + group);
    w.cut = (int32_t*)(base + cut);
    w.part = (float*)(base + part);
    w.part_mz = (float2*)(base + part_mz);
    w.arrived = (uint32_t*)(base + arrived);
    if (ws.base) ctx->paged_kept[ctx->n_paged_kept++] = ws.base;   // kPagedKept times at most (room_for)
    ws = w;
  }
  ws.part_rows = part_rows(max_query_rows);
  ws.max_seqs = max_seqs;
  ws.max_query_rows = max_query_rows;
  ws.max_head_dim = max_head_dim;
  return ASL_OK;
}

asl_status asl_pages_grow(asl_ctx* ctx, const asl_pages* p, const int32_t* rows, const int32_t* add, int32_t n, int32_t* table,
                          int32_t* kv_len, int32_t* refs, void* stream) {
  asl::PageMap m;
  asl_status st = check_pages(ctx, p, table, kv_len, &m);
  if (st == ASL_OK) st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (n == 0) return ASL_OK;
  if (!rows || !add || !refs) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_grow(m, table, kv_len, refs, rows, add, n, ctx->paged.fresh, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "grow launch");
  return ASL_OK;
}

asl_status asl_pages_fork(asl_ctx* ctx, const asl_pages* p, void* const* k_ptrs, void* const* v_ptrs, int32_t n_layers,
                          const int32_t* parents, const int32_t* children, int32_t n, int32_t* table, int32_t* kv_len,
                          int32_t* refs, void* stream) {
  asl::PagesForkArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st == ASL_OK) st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (n_layers < 0) return fail(ctx, ASL_EINVAL, "n_layers must be >= 0");
  if (n_layers > 16384) return fail(ctx, ASL_EUNSUPPORTED, "more than 16384 layers per call");
  if (n == 0) return ASL_OK;
  if (!parents || !children || !refs || (n_layers > 0 && (!k_ptrs || !v_ptrs))) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  const int64_t row_bytes = (int64_t)p->head_dim * elem_bytes(p->dtype);
  if (row_bytes / 16 * p->page_size * p->n_kv_heads > (int64_t(1) << 26))
    return fail(ctx, ASL_EUNSUPPORTED, "pages of more than 2^30 bytes");
  a.table = table;
  a.kv_len = kv_len;
  a.refs = refs;
  a.parents = parents;
  a.children = children;
  a.k_ptrs = k_ptrs;
  a.v_ptrs = v_ptrs;
  a.forks = ctx->paged.forks;
  a.n = n;
  a.n_layers = n_layers;
  a.Hk = p->n_kv_heads;
  set_row_pieces(row_bytes, &a.cpr, &a.cpr_shift);
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_fork(a, ctx->paged.fresh, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "fork launch");
  return ASL_OK;
}

asl_status asl_pages_free(asl_ctx* ctx, const asl_pages* p, const int32_t* rows, int32_t n, const int32_t* table, int32_t* kv_len,
                          int32_t* refs, void* stream) {
  asl::PageMap m;
  asl_status st = check_pages(ctx, p, table, kv_len, &m);
  if (st == ASL_OK) st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (n == 0) return ASL_OK;
  if (!rows || !refs) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_free(m, kv_len, refs, rows, n, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "free launch");
  return ASL_OK;
}

// What asl_pages_write and asl_pages_compact have in common.
static asl_status write_rows(asl_ctx* ctx, const asl_pages* p, asl::PagesWriteArgs& a, const int32_t* rows, const int32_t* cu,
                             int32_t n, int32_t total, const int32_t* idx, int32_t idx_rows, const int32_t* table,
                             const int32_t* kv_len, void* k_pages, void* v_pages, void* stream) {
  asl_status st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (total < 0) return fail(ctx, ASL_EINVAL, "total must be >= 0");
  if (n == 0 || total == 0) return ASL_OK;                 // (tensors without elements have no address)
  if (!rows || !cu || !k_pages || !v_pages || !a.k || !a.v) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  if (a.src_rows && !idx) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  if (idx && idx_rows != 1 && idx_rows != p->n_kv_heads)
    return fail(ctx, ASL_EINVAL, "idx_rows must be 1 or Hk (got %d)", idx_rows);
  if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(ctx, ASL_EUNSUPPORTED, "pages must be 16-byte aligned");
  a.cu = cu;
  a.rows = rows;
  a.idx = idx;
  a.idx_rows = idx_rows;
  a.n = n;
  a.total = total;
  a.k_pages = static_cast<char*>(k_pages);
  a.v_pages = static_cast<char*>(v_pages);
  set_row_pieces((int64_t)p->head_dim * elem_bytes(p->dtype), &a.cpr, &a.cpr_shift);
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_write(a, p->n_kv_heads, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "page write launch");
  return ASL_OK;
}

asl_status asl_pages_write(asl_ctx* ctx, const asl_pages* p, const asl_rows* src, const void* k, const void* v,
                           const int32_t* rows, const int32_t* cu, int32_t n, int32_t total, const int32_t* idx,
                           const int32_t* table, const int32_t* kv_len, void* k_pages, void* v_pages, void* stream) {
  asl::PagesWriteArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st != ASL_OK) return st;
  const char* why = "";
  st = asl::rows_status(*p, src, &why);
  if (st != ASL_OK) return fail(ctx, st, "%s", why);
  if (!aligned16(k) || !aligned16(v)) return fail(ctx, ASL_EUNSUPPORTED, "k and v must be 16-byte aligned");
  const int eb = elem_bytes(p->dtype);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.ksh = src->k_stride_head * eb;
  a.kst = src->k_stride_tok * eb;
  a.vsh = src->v_stride_head * eb;
  a.vst = src->v_stride_tok * eb;
  a.n_src = src->n_src;
  return write_rows(ctx, p, a, rows, cu, n, total, idx, src->idx_rows, table, kv_len, k_pages, v_pages, stream);
}

asl_status asl_pages_compact(asl_ctx* ctx, const asl_pages* p, const int32_t* src_rows, const int32_t* dst_rows, const int32_t* cu,
                             int32_t n, int32_t total, const int32_t* idx, int32_t idx_rows, const int32_t* table,
                             const int32_t* kv_len, void* k_pages, void* v_pages, void* stream) {
  asl::PagesWriteArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st != ASL_OK) return st;
  if (n > 0 && !src_rows) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  a.src_rows = src_rows;
  a.k = static_cast<const char*>(k_pages);
  a.v = static_cast<const char*>(v_pages);
  return write_rows(ctx, p, a, dst_rows, cu, n, total, idx, idx_rows, table, kv_len, k_pages, v_pages, stream);
}

// asl_paged_attention, and with `tree` asl_tree_attention.
static asl_status attend(asl_ctx* ctx, const asl_pages* p, const asl_attn* at, const void* q, const void* k_pages, const void* v_pages,
                         const int32_t* rows, const int32_t* table, const int32_t* kv_len, const int32_t* cu_q, bool tree,
                         const int32_t* parent, const int32_t* group_start, const int32_t* prefix_len, void* out, float* lse,
                         void* stream) {
  asl::AttendArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st != ASL_OK) return st;
  const char* why = "";
  st = asl::attn_status(*p, at, &why);
  if (st == ASL_OK && tree) st = asl::tree_status(*at, &why);
  if (st != ASL_OK) return fail(ctx, st, "%s", why);
  st = check_count(ctx, at->n_seqs);
  if (st != ASL_OK) return st;
  if (p->head_dim > ctx->paged.max_head_dim || (int64_t)at->total_q * p->n_q_heads > ctx->paged.max_query_rows)
    return fail(ctx, ASL_ENOMEM, "total_q*Hq=%lld rows of d=%d exceed what asl_paged_reserve was called for (%d, %d)",
                (long long)at->total_q * p->n_q_heads, p->head_dim, ctx->paged.max_query_rows, ctx->paged.max_head_dim);
  if (at->n_seqs == 0 || at->total_q == 0) return ASL_OK;  // (tensors without elements have no address)
  if (!q || !k_pages || !v_pages || !cu_q || !out || (tree && !parent)) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  if (at->n_groups > 0 && (!group_start || !prefix_len)) return fail(ctx, ASL_EINVAL, "groups need group_start and prefix_len");
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_pages) || !aligned16(v_pages))
    return fail(ctx, ASL_EUNSUPPORTED, "q, out and pages must be 16-byte aligned");
  a.q = q;
  a.k = k_pages;
  a.v = v_pages;
  a.out = out;
  a.lse = lse;
  a.rows = rows;
  a.cu_q = cu_q;
  a.parent = parent;
  a.group_start = at->n_groups > 0 ? group_start : nullptr;
  a.prefix_len = at->n_groups > 0 ? prefix_len : nullptr;
  a.qt = at->q_stride_tok;
  a.qh = at->q_stride_head;
  a.ot = at->out_stride_tok;
  a.oh = at->out_stride_head;
  a.Hq = p->n_q_heads;
  a.Hk = p->n_kv_heads;
  a.G = a.Hq / a.Hk;
  a.d = p->head_dim;
  a.key_bytes = 2 * p->head_dim * elem_bytes(p->dtype) * p->n_kv_heads;
  a.n_seqs = at->n_seqs;
  a.total_q = at->total_q;
  a.max_q_len = at->max_q_len;
  a.max_kv_len = at->max_kv_len;
  a.n_groups = at->n_groups;
  a.causal = (at->flags & ASL_ATTN_CAUSAL) != 0;
  a.scale = p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)p->head_dim);
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e = tree ? asl::launch_attend_tree(ctx->paged, a, p->dtype, s) : asl::launch_attend(ctx->paged, a, p->dtype, s);
  if (e == hipErrorInvalidConfiguration)
    return fail(ctx, ASL_EUNSUPPORTED, "Hk=%d heads of %d sequences and %d query tokens are more than 2^24 work items", p->n_kv_heads, at->n_seqs,
                at->total_q);
  if (e != hipSuccess) return hip_fail(ctx, e, "attention launch");
  return ASL_OK;
}

asl_status asl_paged_attention(asl_ctx* ctx, const asl_pages* p, const asl_attn* at, const void* q, const void* k_pages,
                               const void* v_pages, const int32_t* rows, const int32_t* table, const int32_t* kv_len,
                               const int32_t* cu_q, const int32_t* group_start, const int32_t* prefix_len, void* out, float* lse,
                               void* stream) {
  return attend(ctx, p, at, q, k_pages, v_pages, rows, table, kv_len, cu_q, false, nullptr, group_start, prefix_len, out, lse, stream);
}

asl_status asl_tree_attention(asl_ctx* ctx, const asl_pages* p, const asl_attn* at, const void* q, const void* k_pages,
                              const void* v_pages, const int32_t* rows, const int32_t* table, const int32_t* kv_len,
                              const int32_t* cu_q, const int32_t* parent, const int32_t* group_start, const int32_t* prefix_len,
                              void* out, float* lse, void* stream) {
  return attend(ctx, p, at, q, k_pages, v_pages, rows, table, kv_len, cu_q, true, parent, group_start, prefix_len, out, lse, stream);
}

asl_status asl_pages_plan(asl_ctx* ctx, const asl_pages* p, const int32_t* rows, const int32_t* add, int32_t n, int32_t total,
                          const int32_t* parent, const int32_t* pruned, int32_t* table, int32_t* kv_len, int32_t* refs, int32_t* cu,
                          int64_t* slot, int32_t* pos, void* stream) {
  asl::PlanArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st == ASL_OK) st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (total < 0) return fail(ctx, ASL_EINVAL, "total must be >= 0");
  // (without requests too cu, slot and pos say that there is none: what they held before may be a step's that is over)
  if ((n > 0 && (!rows || !add || !refs)) || !cu || (total > 0 && (!slot || !pos))) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  a.table = table;
  a.kv_len = kv_len;
  a.refs = refs;
  a.rows = rows;
  a.add = add;
  a.parent = parent;
  a.pruned = pruned;
  a.cu = cu;
  a.slot = slot;
  a.pos = pos;
  a.placed = ctx->paged.forks;
  a.fresh = ctx->paged.fresh;
  a.n = n;
  a.total = total;
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_plan(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "plan launch");
  return ASL_OK;
}

asl_status asl_pages_accept(asl_ctx* ctx, const asl_pages* p, void* const* k_ptrs, void* const* v_ptrs, int32_t n_layers,
                            const int32_t* rows, const int32_t* cu, const int32_t* path, int32_t path_stride, const int32_t* n_path,
                            int32_t n, const int64_t* slot, int32_t total, const int32_t* table, int32_t* kv_len, int32_t* refs, void* stream) {
  asl::AcceptArgs a = {};
  asl_status st = check_pages(ctx, p, table, kv_len, &a.map);
  if (st == ASL_OK) st = check_count(ctx, n);
  if (st != ASL_OK) return st;
  if (n_layers < 0 || path_stride < 0 || total < 0) return fail(ctx, ASL_EINVAL, "n_layers, path_stride and total must be >= 0");
  if (n_layers > 16384) return fail(ctx, ASL_EUNSUPPORTED, "more than 16384 layers per call");
  if (path_stride > asl::kTreeNodes) return fail(ctx, ASL_EUNSUPPORTED, "a path of more than %d nodes", asl::kTreeNodes);
  if (n == 0) return ASL_OK;
  if (!rows || !cu || !n_path || !refs || (path_stride > 0 && !path) || (n_layers > 0 && (!k_ptrs || !v_ptrs)))
    return fail(ctx, ASL_EINVAL, "null tensor pointer");
  const int64_t row_bytes = (int64_t)p->head_dim * elem_bytes(p->dtype);
  if (row_bytes / 16 * p->n_kv_heads > (int64_t(1) << 22)) return fail(ctx, ASL_EUNSUPPORTED, "tokens of more than 2^26 bytes");
  a.kv_len = kv_len;
  a.refs = refs;
  a.rows = rows;
  a.cu = cu;
  a.path = path;
  a.n_path = n_path;
  a.slot = slot;                                           // (total 0: a list without entries, of which none is read)
  a.total = total;
  a.k_ptrs = k_ptrs;
  a.v_ptrs = v_ptrs;
  a.arrived = ctx->paged.arrived;
  a.n = n;
  a.path_stride = path_stride;
  a.n_layers = n_layers;
  a.Hk = p->n_kv_heads;
  set_row_pieces(row_bytes, &a.cpr, &a.cpr_shift);
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_pages_accept(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "accept launch");
  return ASL_OK;
}

asl_status asl_rotation_freqs(const asl_freqs* freqs, double* out) { return asl::rotation_freqs(freqs, out); }

// What asl_rotate and asl_rotate_write have in common; a has what only one of them does.
static asl_status rotate(asl_ctx* ctx, const asl_rotation* r, asl::RotateArgs& a, const void* q, const void* k, const int32_t* pos,
                         const double* freqs, int32_t n, void* q_out, bool write, void* stream) {
  if (n < 0) return fail(ctx, ASL_EINVAL, "the number of tokens must be >= 0");
  if (n == 0 || (r->n_q_heads == 0 && r->n_kv_heads == 0)) return ASL_OK;
  if (!pos || !freqs || (r->n_q_heads > 0 && (!q || !q_out)) || (r->n_kv_heads > 0 && (!k || !a.k_out)))
    return fail(ctx, ASL_EINVAL, "null tensor pointer");
  auto one_place = [n](int heads, int64_t tok, int64_t head) { return (heads > 0 && n > 1 && tok == 0) || (heads > 1 && head == 0); };
  if (one_place(r->n_q_heads, r->q_out_stride_tok, r->q_out_stride_head) ||
      (!write && one_place(r->n_kv_heads, r->k_out_stride_tok, r->k_out_stride_head)))
    return fail(ctx, ASL_EINVAL, "outputs of several tokens or heads in one place (a stride of 0)");
  const int eb = elem_bytes(r->dtype);
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.q_out = static_cast<char*>(q_out);
  a.pos = pos;
  a.freqs = freqs;
  a.qt = r->q_stride_tok * eb;
  a.qh = r->q_stride_head * eb;
  a.kt = r->k_stride_tok * eb;
  a.kh = r->k_stride_head * eb;
  a.vt = r->v_stride_tok * eb;
  a.vh = r->v_stride_head * eb;
  a.qot = r->q_out_stride_tok * eb;
  a.qoh = r->q_out_stride_head * eb;
  a.kot = r->k_out_stride_tok * eb;
  a.koh = r->k_out_stride_head * eb;
  a.n = n;
  a.Hq = r->n_q_heads;
  a.Hk = r->n_kv_heads;
  a.d = r->head_dim;
  a.rot = r->rot_dim;
  const float by = r->magnitude > 0.f ? r->magnitude : 1.f;
  a.cos_by = by;
  a.sin_by = (r->flags & ASL_ROTATE_BACK) != 0 ? -by : by;
  a.in_place = !write && (a.Hq == 0 || (a.q == a.q_out && a.qt == a.qot && a.qh == a.qoh)) &&
               (a.Hk == 0 || (a.k == a.k_out && a.kt == a.kot && a.kh == a.koh));
  // the bits that any address or stride has set
  uint64_t bits = 0;
  if (a.Hq > 0) bits |= (uint64_t)a.q | (uint64_t)a.q_out | (uint64_t)(a.qt | a.qh | a.qot | a.qoh);
  if (a.Hk > 0) bits |= (uint64_t)a.k | (uint64_t)a.k_out | (uint64_t)(a.kt | a.kh);
  if (a.Hk > 0 && !write) bits |= (uint64_t)(a.kot | a.koh);
  if (a.Hk > 0 && write) bits |= (uint64_t)a.v | (uint64_t)a.v_out | (uint64_t)(a.vt | a.vh);
  if (bits % eb != 0) return fail(ctx, ASL_EUNSUPPORTED, "tensors must be aligned to their elements");
  const int width = asl::rotate_width(*r, bits % 16 == 0 ? 16 : (int64_t)(bits & (~bits + 1)));
  DeviceGuard guard(ctx->device);
  if (guard.err != hipSuccess) return hip_fail(ctx, guard.err, "set device");
  hipError_t e = asl::launch_rotate(a, r->dtype, r->pairs == ASL_PAIRS_HALVES, write, width, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(ctx, e, "rotation launch");
  return ASL_OK;
}

asl_status asl_rotate(asl_ctx* ctx, const asl_rotation* r, const void* q, const void* k, const int32_t* pos, const double* freqs, int32_t n,
                      void* q_out, void* k_out, void* stream) {
  if (!ctx) return ASL_EINVAL;
  const char* why = "";
  const asl_status st = asl::rotation_status(r, &why);
  if (st != ASL_OK) return fail(ctx, st, "%s", why);
  asl::RotateArgs a = {};
  a.k_out = static_cast<char*>(k_out);
  return rotate(ctx, r, a, q, k, pos, freqs, n, q_out, false, stream);
}

asl_status asl_rotate_write(asl_ctx* ctx, const asl_pages* p, const asl_rotation* r, const void* q, const void* k, const void* v,
                            const int32_t* pos, const int64_t* slot, const double* freqs, int32_t n, void* q_out, void* k_pages,
                            void* v_pages, void* stream) {
  if (!ctx) return ASL_EINVAL;
  const char* why = "";
  asl_status st = asl::pages_status(p, &why);
  if (st == ASL_OK) st = asl::rotation_status(r, &why);
  if (st != ASL_OK) return fail(ctx, st, "%s", why);
  if (!ctx->paged.base) return fail(ctx, ASL_ENOMEM, "call asl_paged_reserve first");
  if (r->n_kv_heads != p->n_kv_heads || r->head_dim != p->head_dim || r->dtype != p->dtype)
    return fail(ctx, ASL_EINVAL, "rotation and pages differ in KV heads, head_dim or dtype");
  asl::RotateArgs a = {};
  if (n > 0 && (!v || !slot || !v_pages)) return fail(ctx, ASL_EINVAL, "null tensor pointer");
  if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(ctx, ASL_EUNSUPPORTED, "pages must be 16-byte aligned");
  a.map = asl::page_map(*p, elem_bytes(p->dtype), nullptr, nullptr, ctx->paged.fault);
  a.slot = slot;
  a.v = static_cast<const char*>(v);
  a.k_out = static_cast<char*>(k_pages);
  a.v_out = static_cast<char*>(v_pages);
  return rotate(ctx, r, a, q, k, pos, freqs, n, q_out, true, stream);
}

#pragma GCC visibility pop
}  // extern "C"
