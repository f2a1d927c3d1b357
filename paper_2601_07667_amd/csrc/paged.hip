// The pages of a cache: writing tokens into them, compacting, growing, forking and freeing sequences.
//
// Which pages are free is said by the counts alone (0 = free), and a call takes the lowest-numbered free pages in the order of its
// list: results do not depend on timing, and nothing has to be kept beside the counts.  Looking for the pages reads counts until
// enough are found, at most 4 bytes a page (a pool of 64K pages: 256 KB).
#include "paged.h"

#include "asl_internal.h"

namespace asl {

namespace {

constexpr int kWriteThreads = 256;
constexpr int kBookThreads = 1024;

__device__ __forceinline__ void paged_fault(const PageMap& m) { atomicOr(m.fault, kFaultPaged); }

// Rows of head_dim elements into the last cu[i + 1] - cu[i] positions of table row rows[i], for every i: a copy, bound by memory.
// Each thread moves U pieces of 16 bytes; the pieces of a (head, tensor) are numbered token * cpr + c, so a wavefront reads and
// writes whole rows.  PAGED: the source is a row's pages too.  grid: x = blocks of pieces, y = KV head, z = K or V.
template <bool PAGED, int U>
__global__ void __launch_bounds__(kWriteThreads) pages_write_kernel(PagesWriteArgs a) {
  typedef uint32_t Piece __attribute__((ext_vector_type(4)));
  extern __shared__ int32_t cu[];
  for (int i = threadIdx.x; i <= a.n; i += kWriteThreads) cu[i] = a.cu[i];
  __syncthreads();
  const int h = blockIdx.y, which = blockIdx.z;
  const char* src = which == 0 ? a.k : a.v;
  char* dst = (which == 0 ? a.k_pages : a.v_pages) + (int64_t)h * a.map.head;
  const int64_t sh = which == 0 ? a.ksh : a.vsh, stt = which == 0 ? a.kst : a.vst;
  src += PAGED ? (int64_t)h * a.map.head : (int64_t)h * sh;
  const int32_t* idx = a.idx != nullptr ? a.idx + (a.idx_rows == 1 ? 0 : (int64_t)h * a.total) : nullptr;
  const int64_t total = (int64_t)a.total * a.cpr;
  const int64_t q0 = (int64_t)blockIdx.x * (kWriteThreads * U) + threadIdx.x;
  Piece val[U];
  int64_t to[U];
  bool bad = false;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    to[u] = -1;
    const int64_t q = q0 + u * kWriteThreads;
    if (q >= total) continue;
    const int j = a.cpr_shift >= 0 ? (int)(q >> a.cpr_shift) : (int)(q / a.cpr);
    const int c = (int)(q - (int64_t)j * a.cpr);
    const int i = sequence_of(cu, a.n, j);
    const int t = idx != nullptr ? idx[j] : j;
    const int r = a.rows[i];
    int64_t from = -1;
    if (PAGED) {
      const int rs = a.src_rows[i];
      int len;
      if (row_length(a.map, rs, &len) && t < len) from = token_offset(a.map, rs, t);
    } else if ((uint32_t)t < (uint32_t)a.n_src) {
      from = (int64_t)t * stt;
    }
    int64_t at = -1;
    int len;
    if (cu[i] <= j && j < cu[i + 1] && row_length(a.map, r, &len)) at = token_offset(a.map, r, len - (cu[i + 1] - j));
    if (from < 0 || at < 0) {
      bad = true;
      continue;
    }
    to[u] = at + c * 16;
    val[u] = *(const Piece*)(src + from + c * 16);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (to[u] >= 0) *(Piece*)(dst + to[u]) = val[u];
  if (bad) paged_fault(a.map);
}

// ---------------------------------------------------------------------------------------------------------------------
// Bookkeeping, by one workgroup of kBookThreads.

struct BookLds {
  int32_t incl[kPagedMaxSeqs];             // pages needed by the requests up to each, itself among them
  int32_t wave[kBookThreads / 64];
  int32_t found;
};

// Inclusive prefix sum over the workgroup; *total gets the sum.
__device__ __forceinline__ int block_scan(int x, BookLds& l, int* total) {
  const int wave = threadIdx.x >> 6;
  const int own = (int)wave_prefix_sum((uint32_t)x);
  __syncthreads();                         // the last reader of l.wave is done
  if ((threadIdx.x & 63) == 63) l.wave[wave] = own;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kBookThreads / 64; ++w) {
    const int s = l.wave[w];
    before += w < wave ? s : 0;
    all += s;
  }
  *total = all;
  return before + own;
}

// l.incl[i] = needs[0] + .. + needs[i] of n requests (each at most kMaxFresh + 1), thread t holding those of i = t + 1024 u;
// returns the sum.
__device__ __forceinline__ int scan_needs(const int (&need)[kPagedMaxSeqs / kBookThreads], int n, BookLds& l) {
  int base = 0;
#pragma unroll
  for (int u = 0; u < kPagedMaxSeqs / kBookThreads; ++u) {
    if (u * kBookThreads >= n) break;
    int total;
    const int incl = block_scan(need[u], l, &total);
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i < n) l.incl[i] = base + incl;
    base += total;
  }
  __syncthreads();
  return base;
}

// The first `want` pages whose count is 0, in order, to fresh[]; returns how many there are (at most `want`).
__device__ __forceinline__ int find_free(const int32_t* refs, int n_pages, int want, int32_t* fresh, BookLds& l) {
  constexpr int PER = 8;
  int base = 0;
  for (int64_t p0 = 0; p0 < n_pages && base < want; p0 += kBookThreads * PER) {
    const int64_t p = p0 + (int64_t)threadIdx.x * PER;
    uint32_t free = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (p + k < n_pages && refs[p + k] == 0) free |= 1u << k;
    int total;
    int at = base + block_scan(__popc(free), l, &total) - __popc(free);
    while (free != 0 && at < want) {
      fresh[at++] = (int32_t)p + __ffs(free) - 1;
      free &= free - 1;
    }
    base += total;
  }
  __syncthreads();
  return min(base, want);
}

// Row r's length while a request of this call has it: marks it, so that a second request for the same row finds it taken.
__device__ __forceinline__ bool take_row(int32_t* kv_len, int r, int len) {
  return atomicCAS(&kv_len[r], len, -1 - len) == len;
}

__global__ void __launch_bounds__(kBookThreads)
pages_grow_kernel(PageMap m, int32_t* table, int32_t* kv_len, int32_t* refs, const int32_t* rows, const int32_t* add, int n,
                  int32_t* fresh) {
  __shared__ BookLds l;
  constexpr int UN = kPagedMaxSeqs / kBookThreads;
  int row[UN], len[UN], more[UN], need[UN];
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    row[u] = -1;
    len[u] = more[u] = need[u] = 0;
    if (i >= n) continue;
    const int r = rows[i], x = add[i];
    if ((uint32_t)r >= (uint32_t)m.n_rows || x < 0) { paged_fault(m); continue; }
    const int old = kv_len[r];
    if (old < 0 || (int64_t)old + x > (int64_t)m.row_stride * m.ps || !take_row(kv_len, r, old)) { paged_fault(m); continue; }
    row[u] = r;
    len[u] = old;
    more[u] = x;
    need[u] = min((int)(((int64_t)old + x + m.ps - 1) >> m.ps_shift) - (int)(((int64_t)old + m.ps - 1) >> m.ps_shift),
                  kMaxFresh + 1);
  }
  const int want = min(scan_needs(need, n, l), kMaxFresh);
  const int got = find_free(refs, m.n_pages, want, fresh, l);
  // every fresh page to the request that its number falls to
  for (int k = threadIdx.x; k < got; k += kBookThreads) {
    int lo = -1, hi = n - 1;                               // incl[lo] <= k < incl[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (l.incl[mid] <= k) lo = mid; else hi = mid;
    }
    if (l.incl[hi] > got) continue;                        // the request does not get all that it needs, so it gets nothing
    const int r = rows[hi], before = hi > 0 ? l.incl[hi - 1] : 0;
    const int old = -1 - __hip_atomic_load(&kv_len[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // as marked
    table[(int64_t)r * m.row_stride + ((int64_t)(old + m.ps - 1) >> m.ps_shift) + (k - before)] = fresh[k];
    refs[fresh[k]] = 1;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < UN; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i < n && row[u] >= 0) kv_len[row[u]] = l.incl[i] <= got ? len[u] + more[u] : len[u];
  }
}

// Which page each continuation gets for the parent's last, partly filled one: forks[i] = (parent, child, length, page), length 0
// where there is nothing to do, page -1 where the parent fills its last page.
__global__ void __launch_bounds__(kBookThreads) pages_fork_kernel(PagesForkArgs a, int32_t* fresh) {
  __shared__ BookLds l;
  constexpr int UN = kPagedMaxSeqs / kBookThreads;
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

// The continuations' rows and counts (slice 0), and the filled tokens of their last pages (slices from 1: layer, K or V).
__global__ void __launch_bounds__(kWriteThreads) pages_fork_copy_kernel(PagesForkArgs a) {
  typedef uint32_t Piece __attribute__((ext_vector_type(4)));
  const PageMap& m = a.map;
  const int4 f = a.forks[blockIdx.x];
  if (f.z <= 0) return;
  const int full = f.z >> m.ps_shift, part = f.z & (m.ps - 1);
  const int32_t* from = m.table + (int64_t)f.x * m.row_stride;
  if (blockIdx.y == 0) {
    int32_t* to = a.table + (int64_t)f.y * m.row_stride;
    bool bad = false;
    for (int t = threadIdx.x; t < full; t += kWriteThreads) {
      const int page = from[t];
      to[t] = page;
      if ((uint32_t)page < (uint32_t)m.n_pages) atomicAdd(&a.refs[page], 1); else bad = true;
    }
    if (threadIdx.x == 0 && part != 0) to[full] = f.w;
    if (bad) paged_fault(m);
    return;
  }
  if (part == 0) return;
  const int slice = (int)blockIdx.y - 1, layer = slice >> 1;
  char* base = (char*)((slice & 1) == 0 ? a.k_ptrs[layer] : a.v_ptrs[layer]);
  const int page = from[full];
  if ((uint32_t)page >= (uint32_t)m.n_pages) {
    if (threadIdx.x == 0) paged_fault(m);
    return;
  }
  const int per_head = part * a.cpr, total = per_head * a.Hk;
  for (int q = threadIdx.x; q < total; q += kWriteThreads) {
    const int h = q / per_head, e = q - h * per_head;
    const int t = a.cpr_shift >= 0 ? e >> a.cpr_shift : e / a.cpr;
    const int64_t off = (int64_t)h * m.head + (int64_t)t * m.tok + (int64_t)(e - t * a.cpr) * 16;
    *(Piece*)(base + (int64_t)f.w * m.page + off) = *(const Piece*)(base + (int64_t)page * m.page + off);
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

hipError_t launch_pages_write(const PagesWriteArgs& a, int Hk, hipStream_t st) {
  if (a.n == 0 || a.total == 0) return hipSuccess;
  const size_t lds = (size_t)(a.n + 1) * sizeof(int32_t);
  const int64_t pieces = (int64_t)a.total * a.cpr;
  const int64_t blocks = (pieces + kWriteThreads * 4 - 1) / (kWriteThreads * 4);
  if (blocks >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks, (unsigned)Hk, 2);
  if (a.src_rows != nullptr)
    hipLaunchKernelGGL((pages_write_kernel<true, 4>), grid, dim3(kWriteThreads), lds, st, a);
  else
    hipLaunchKernelGGL((pages_write_kernel<false, 4>), grid, dim3(kWriteThreads), lds, st, a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesForkArgs& a, int32_t* fresh, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(pages_fork_kernel, dim3(1), dim3(kBookThreads), 0, st, a, fresh);
  hipLaunchKernelGGL(pages_fork_copy_kernel, dim3((unsigned)a.n, (unsigned)(1 + 2 * a.n_layers)), dim3(kWriteThreads), 0, st, a);
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
