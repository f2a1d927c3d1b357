// The pages of a cache: writing tokens into them, compacting, growing, forking and freeing sequences.
//
// Which pages are free is said by the counts alone (0 = free), and a call takes the lowest-numbered free pages in the order of its
// list: results do not depend on timing, and nothing has to be kept beside the counts.  Looking for the pages reads counts until
// enough are found, at most 4 bytes a page (a pool of 64K pages: 256 KB).
#include "paged.h"

#include "asl_internal.h"
#include "pages_book.h"

namespace asl {

namespace {

constexpr int kWriteThreads = 256;

typedef uint32_t Piece __attribute__((ext_vector_type(4)));              // 16 bytes
typedef const Piece __attribute__((address_space(1))) * PieceSrc;
typedef Piece __attribute__((address_space(1))) * PieceDst;

// STREAM: past the caches (transfers that do not fit them anyway).
template <bool STREAM>
__device__ __forceinline__ Piece load_piece(const char* p) {
  return STREAM ? __builtin_nontemporal_load((PieceSrc)p) : *(PieceSrc)p;
}
template <bool STREAM>
__device__ __forceinline__ void store_piece(char* p, Piece x) {
  if (STREAM) __builtin_nontemporal_store(x, (PieceDst)p); else *(PieceDst)p = x;
}

constexpr int kWriteUnroll = 4;            // pieces of K, and as many of V, that a thread has on their way
constexpr int kWriteTokens = kWriteThreads;   // most tokens of a workgroup
constexpr int kWriteStaged = 1024;         // sequences whose rows and lengths a workgroup takes to LDS (at most 20 KB) rather than look them up

// Rows of head_dim elements into the last cu[i + 1] - cu[i] positions of table row rows[i], for every i: a copy, bound by memory.
// A workgroup has some neighbouring tokens of a KV head: first a thread for each finds where it stands and where it goes (sequence,
// row, length, page: loads that depend on each other), then all move the tokens' pieces of 16 bytes, K and V, numbered
// token * cpr + c, so that a wavefront reads and writes whole rows.  PAGED: the source is a row's pages too.
// grid: x = blocks of a.tokens tokens, y = KV head.
template <bool PAGED, bool STREAM>
__global__ void __launch_bounds__(kWriteThreads) pages_write_kernel(PagesWriteArgs a) {
  extern __shared__ int32_t lds[];         // cu [n + 1]; staged: rows [n], lengths [n] of the rows written to, then of those read
  __shared__ int64_t from[kWriteTokens], to[kWriteTokens];               // byte offsets within the head's source and pages; to -1: none
  int32_t* cu = lds;
  int32_t* row = lds + a.n + 1;
  int32_t* len = row + a.n;
  int32_t* src_row = len + a.n;
  int32_t* src_len = src_row + a.n;
  const int h = blockIdx.y, tid = threadIdx.x;
  const int j0 = (int)blockIdx.x * a.tokens, n_tok = min(a.tokens, a.total - j0);
  const int32_t* idx = a.idx != nullptr ? a.idx + (a.idx_rows == 1 ? 0 : (int64_t)h * a.total) : nullptr;
  const int t = tid < n_tok ? (idx != nullptr ? idx[j0 + tid] : j0 + tid) : 0;
  bool bad = false;
  const bool staged = a.n <= kWriteStaged;
  for (int i = tid; i <= a.n; i += kWriteThreads) {
    cu[i] = a.cu[i];
    if (staged && i < a.n) {
      const int r = a.rows[i];
      int L;
      row[i] = row_length(a.map, r, &L) ? r : -1;
      len[i] = L;
      if (PAGED) {
        const int rs = a.src_rows[i];
        src_row[i] = row_length(a.map, rs, &L) ? rs : -1;
        src_len[i] = L;
      }
    }
  }
  __syncthreads();
  if (tid < n_tok) {
    const int j = j0 + tid, i = sequence_of(cu, a.n, j);
    int64_t f = -1, w = -1;
    int r, L, rs = -1, Ls = 0;
    if (staged) {
      r = row[i];
      L = len[i];
      if (PAGED) {
        rs = src_row[i];
        Ls = src_len[i];
      }
    } else {
      r = row_length(a.map, a.rows[i], &L) ? a.rows[i] : -1;
      if (PAGED) rs = row_length(a.map, a.src_rows[i], &Ls) ? a.src_rows[i] : -1;
    }
    if (PAGED) {
      if (t < Ls) f = token_offset(a.map, rs, t);          // t < 0: -1 as well
    } else if ((uint32_t)t < (uint32_t)a.n_src) {
      f = t;
    }
    if (cu[i] <= j && j < cu[i + 1]) w = token_offset(a.map, r, L - (cu[i + 1] - j));
    bad = f < 0 || w < 0;
    from[tid] = f;
    to[tid] = bad ? -1 : w;
  }
  __syncthreads();
  const int64_t head = (int64_t)h * a.map.head;
  const char* ks = a.k + (PAGED ? head : (int64_t)h * a.ksh);
  const char* vs = a.v + (PAGED ? head : (int64_t)h * a.vsh);
  const int pieces = n_tok * a.cpr;
  for (int q0 = tid; q0 < pieces; q0 += kWriteThreads * kWriteUnroll) {
    Piece k[kWriteUnroll], v[kWriteUnroll];
    int64_t at[kWriteUnroll];
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
      const int q = q0 + u * kWriteThreads;
      at[u] = -1;
      if (q >= pieces) continue;
      const int j = a.cpr_shift >= 0 ? q >> a.cpr_shift : (int)((uint32_t)q / (uint32_t)a.cpr);
      const int c = (q - j * a.cpr) * 16;
      if (to[j] < 0) continue;
      at[u] = head + to[j] + c;
      k[u] = load_piece<STREAM>(ks + (PAGED ? from[j] : from[j] * a.kst) + c);
      v[u] = load_piece<STREAM>(vs + (PAGED ? from[j] : from[j] * a.vst) + c);
    }
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u)
      if (at[u] >= 0) {
        store_piece<STREAM>(a.k_pages + at[u], k[u]);
        store_piece<STREAM>(a.v_pages + at[u], v[u]);
      }
  }
  if (bad) paged_fault(a.map);
}

// ---------------------------------------------------------------------------------------------------------------------
// Bookkeeping, by one workgroup of kBookThreads (pages_book.h).

__global__ void __launch_bounds__(kBookThreads)
pages_grow_kernel(PageMap m, int32_t* table, int32_t* kv_len, int32_t* refs, const int32_t* rows, const int32_t* add, int n,
                  int32_t* fresh) {
  __shared__ BookLds l;
  Growth g[kBookUnroll];
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i < n && !g[u].take(m, kv_len, rows[i], add[i])) paged_fault(m);
  }
  give_pages(m, table, kv_len, refs, rows, n, fresh, g, l);
}

// Which page each continuation gets for the parent's last, partly filled one: forks[i] = (parent, child, length, page), length 0
// where there is nothing to do, page -1 where the parent fills its last page.
__global__ void __launch_bounds__(kBookThreads) pages_fork_kernel(PagesForkArgs a, int32_t* fresh) {
  __shared__ BookLds l;
  constexpr int UN = kBookUnroll;
  const PageMap& m = a.map;
  int parent[UN], child[UN], len[UN], need[UN];
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    parent[u] = child[u] = -1;
    len[u] = need[u] = 0;
    if (i >= a.n) continue;
    const int p = a.parents[i], c = a.children[i];
    if ((uint32_t)p >= (uint32_t)m.n_rows || (uint32_t)c >= (uint32_t)m.n_rows) { paged_fault(m); continue; }
    const int L = a.kv_len[p];
    if (L < 0 || L > (int64_t)m.row_stride * m.ps) { paged_fault(m); continue; }
    parent[u] = p;
    child[u] = c;
    len[u] = L;
  }
  __syncthreads();                                         // every length is read before the first row is marked
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    if (child[u] < 0) continue;
    if (!take_row(a.kv_len, child[u], 0)) {                // not empty, or named twice
      paged_fault(m);
      child[u] = -1;
      len[u] = 0;
    }
    need[u] = (len[u] & (m.ps - 1)) != 0 ? 1 : 0;
  }
  const int want = min(scan_needs(need, a.n, l), kMaxFresh);
  const int got = find_free(a.refs, m.n_pages, want, fresh, l);
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i >= a.n) continue;
    const bool fits = child[u] >= 0 && l.incl[i] <= got;
    int page = -1;
    if (fits && need[u]) {
      page = fresh[l.incl[i] - 1];
      a.refs[page] = 1;
    }
    if (child[u] >= 0) a.kv_len[child[u]] = fits ? len[u] : 0;
    a.forks[i] = make_int4(parent[u], child[u], fits ? len[u] : 0, page);
  }
}

// The continuations' rows and counts (slice 0), and the filled tokens of their last pages (slices from 1: layer, K or V), kForkGroup
// neighbouring continuations a workgroup.  grid: x = groups, y = slices, z = blocks of kForkPieces pieces of the page.  Neighbours mostly
// have one parent: its pieces are read once and stored for each of them (24 parents continued 8 times, 16 layers: 136 us with a
// workgroup for each continuation).
constexpr int kForkGroup = 8;
constexpr int kForkUnroll = 8;             // pieces of a thread
constexpr int kForkPieces = kWriteThreads * kForkUnroll;
__global__ void __launch_bounds__(kWriteThreads) pages_fork_copy_kernel(PagesForkArgs a) {
  const PageMap& m = a.map;
  const int i0 = (int)blockIdx.x * kForkGroup, count = min(kForkGroup, a.n - i0);
  __shared__ int4 forks[kForkGroup];
  __shared__ int32_t last[kForkGroup];     // the parent's last, partly filled page, or -1
  if ((int)threadIdx.x < count) {
    const int4 f = a.forks[i0 + threadIdx.x];
    forks[threadIdx.x] = f;
    int page = -1;
    if (f.z > 0 && f.w >= 0) {
      page = m.table[(int64_t)f.x * m.row_stride + (f.z >> m.ps_shift)];
      if ((uint32_t)page >= (uint32_t)m.n_pages) {
        page = -1;
        paged_fault(m);
      }
    }
    last[threadIdx.x] = page;
  }
  __syncthreads();
  if (blockIdx.y == 0) {
    if (blockIdx.z != 0) return;
    bool bad = false;
    for (int i = 0; i < count; ++i) {
      const int4 f = forks[i];
      if (f.z <= 0) continue;
      const int full = f.z >> m.ps_shift;
      const int32_t* from = m.table + (int64_t)f.x * m.row_stride;
      int32_t* to = a.table + (int64_t)f.y * m.row_stride;
      for (int t = threadIdx.x; t < full; t += kWriteThreads) {
        const int page = from[t];
        to[t] = page;
        if ((uint32_t)page < (uint32_t)m.n_pages) atomicAdd(&a.refs[page], 1); else bad = true;
      }
      if (threadIdx.x == 0 && f.w >= 0) to[full] = f.w;
    }
    if (bad) paged_fault(m);
    return;
  }
  const int slice = (int)blockIdx.y - 1, layer = slice >> 1;
  char* base = (char*)((slice & 1) == 0 ? a.k_ptrs[layer] : a.v_ptrs[layer]);
  const uint32_t q0 = blockIdx.z * (uint32_t)kForkPieces + threadIdx.x;
  Piece x[kForkUnroll];
  int64_t off[kForkUnroll];
  int parent = -1;
  for (int i = 0; i < count; ++i) {
    const int4 f = forks[i];
    const int page = last[i];
    if (page < 0) continue;
    const uint32_t per_head = (uint32_t)(f.z & (m.ps - 1)) * (uint32_t)a.cpr, total = per_head * (uint32_t)a.Hk;
    if (f.x != parent) {
      parent = f.x;
      const char* src = base + (int64_t)page * m.page;
#pragma unroll
      for (int u = 0; u < kForkUnroll; ++u) {
        const uint32_t q = min(q0 + u * kWriteThreads, total - 1u), h = q / per_head, e = q - h * per_head;
        const uint32_t t = a.cpr_shift >= 0 ? e >> a.cpr_shift : e / (uint32_t)a.cpr;
        off[u] = (int64_t)h * m.head + (int64_t)t * m.tok + (int64_t)(e - t * (uint32_t)a.cpr) * 16;
        x[u] = load_piece<false>(src + off[u]);
      }
    }
    char* dst = base + (int64_t)f.w * m.page;
#pragma unroll
    for (int u = 0; u < kForkUnroll; ++u)
      if (q0 + u * kWriteThreads < total) store_piece<true>(dst + off[u], x[u]);
  }
}

// One workgroup a row: its pages' counts go down by one, its length to 0.
__global__ void __launch_bounds__(kWriteThreads)
pages_free_kernel(PageMap m, int32_t* kv_len, int32_t* refs, const int32_t* rows, int n) {
  __shared__ int32_t len;
  const int r = rows[blockIdx.x];
  if (threadIdx.x == 0) {
    len = 0;
    if ((uint32_t)r >= (uint32_t)m.n_rows) {
      paged_fault(m);
    } else {
      const int old = atomicExch(&kv_len[r], 0);           // a row that is named twice is freed once
      if (old >= 0 && old <= (int64_t)m.row_stride * m.ps) len = old; else paged_fault(m);
    }
  }
  __syncthreads();
  const int pages = (len + m.ps - 1) >> m.ps_shift;
  bool bad = false;
  for (int t = threadIdx.x; t < pages; t += kWriteThreads) {
    const int page = m.table[(int64_t)r * m.row_stride + t];
    if ((uint32_t)page >= (uint32_t)m.n_pages) {
      bad = true;
    } else if (atomicSub(&refs[page], 1) <= 0) {           // nobody held it
      atomicAdd(&refs[page], 1);
      bad = true;
    }
  }
  if (bad) paged_fault(m);
}

}  // namespace

// Bytes read and written from which pages are written past the caches (gather.hip has the measurement of the same copy).
constexpr int64_t kWriteStreamBytes = int64_t(100) << 20;

hipError_t launch_pages_write(const PagesWriteArgs& args, int Hk, hipStream_t st) {
  PagesWriteArgs a = args;
  if (a.n == 0 || a.total == 0) return hipSuccess;
  // a workgroup has pieces for one round of its threads; fewer tokens where the call does not fill the card
  const int round = kWriteThreads * kWriteUnroll / a.cpr;
  a.tokens = round < 1 ? 1 : round > kWriteTokens ? kWriteTokens : round;
  while (a.tokens > 8 && (int64_t)(a.total / a.tokens + 1) * Hk < 256) a.tokens /= 2;
  const int64_t blocks = ((int64_t)a.total + a.tokens - 1) / a.tokens;
  const size_t lds = (size_t)(a.n + 1 + (a.n > kWriteStaged ? 0 : (a.src_rows != nullptr ? 4 : 2) * a.n)) * sizeof(int32_t);
  const bool stream = 4 * (int64_t)a.total * a.cpr * 16 * Hk >= kWriteStreamBytes;
  const dim3 grid((unsigned)blocks, (unsigned)Hk), block(kWriteThreads);
  if (a.src_rows != nullptr && stream)
    hipLaunchKernelGGL((pages_write_kernel<true, true>), grid, block, lds, st, a);
  else if (a.src_rows != nullptr)
    hipLaunchKernelGGL((pages_write_kernel<true, false>), grid, block, lds, st, a);
  else if (stream)
    hipLaunchKernelGGL((pages_write_kernel<false, true>), grid, block, lds, st, a);
  else
    hipLaunchKernelGGL((pages_write_kernel<false, false>), grid, block, lds, st, a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesForkArgs& a, int32_t* fresh, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(kBookThreads), 0, st, a, fresh);
  const int64_t pieces = (int64_t)(a.map.ps - 1) * a.cpr * a.Hk;   // at most 2^26 (asl_pages_fork)
  const dim3 grid((unsigned)((a.n + kForkGroup - 1) / kForkGroup), (unsigned)(1 + 2 * a.n_layers),
                  (unsigned)((pieces + kForkPieces - 1) / kForkPieces));
  hipLaunchKernelGGL(pages_fork_copy_kernel, grid, dim3(kWriteThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_pages_grow(const PageMap& map, int32_t* table, int32_t* kv_len, int32_t* refs, const int32_t* rows,
                             const int32_t* add, int n, int32_t* fresh, hipStream_t st) {
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(pages_grow_kernel, dim3(1), dim3(kBookThreads), 0, st, map, table, kv_len, refs, rows, add, n, fresh);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PageMap& map, int32_t* kv_len, int32_t* refs, const int32_t* rows, int n, hipStream_t st) {
  if (n == 0) return hipSuccess;
  hipLaunchKernelGGL(pages_free_kernel, dim3((unsigned)n), dim3(kWriteThreads), 0, st, map, kv_len, refs, rows, n);
  return hipGetLastError();
}

}  // namespace asl
