// The bookkeeping of pages, by one workgroup of kBookThreads: which free pages the requests of a call get.
//
// Requests are served in the order of the list, with the lowest-numbered free pages; the first that does not get all that it needs, and all
// behind it, get none.  Thread t has requests t, t + 1024, ...
#pragma once
#include "paged.h"

#include "asl_internal.h"

namespace asl {

namespace {

constexpr int kBookThreads = 1024;
constexpr int kBookUnroll = kPagedMaxSeqs / kBookThreads;      // requests of a thread

__device__ __forceinline__ void paged_fault(const PageMap& m) { atomicOr(m.fault, kFaultPaged); }

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
__device__ __forceinline__ int scan_needs(const int (&need)[kBookUnroll], int n, BookLds& l) {
  int base = 0;
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
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
  constexpr int PER = 16;                  // pages of a thread and round: 64K pages take four
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

// A request: row `row` (-1: none, or out of range) of len tokens is to hold `more` more, for which it needs so many pages.
struct Growth {
  int row = -1, len = 0, more = 0, need = 0;

  // Reads request (r, x) and marks the row; false, and nothing is done, if it is out of range or another request has the row.
  __device__ __forceinline__ bool take(const PageMap& m, int32_t* kv_len, int r, int x) {
    if ((uint32_t)r >= (uint32_t)m.n_rows || x < 0) return false;
    const int old = kv_len[r];
    if (old < 0 || (int64_t)old + x > (int64_t)m.row_stride * m.ps || !take_row(kv_len, r, old)) return false;
    row = r;
    len = old;
    more = x;
    need = min((int)(((int64_t)old + x + m.ps - 1) >> m.ps_shift) - (int)(((int64_t)old + m.ps - 1) >> m.ps_shift), kMaxFresh + 1);
    return true;
  }
};

// Pages for the rows that the requests have marked, and their new lengths.  Returns how many pages there were: request i got its own iff
// l.incl[i] is not more.
__device__ __forceinline__ int give_pages(const PageMap& m, int32_t* table, int32_t* kv_len, int32_t* refs, const int32_t* rows, int n,
                                          int32_t* fresh, const Growth (&g)[kBookUnroll], BookLds& l) {
  int need[kBookUnroll];
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) need[u] = g[u].need;
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
  for (int u = 0; u < kBookUnroll; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i < n && g[u].row >= 0) kv_len[g[u].row] = l.incl[i] <= got ? g[u].len + g[u].more : g[u].len;
  }
  return got;
}

}  // namespace

}  // namespace asl
