// Drafting over the paged cache: the plan of a batch (asl_pages_plan) and the path that is kept of a draft (asl_pages_accept).
#include "paged.h"

#include "asl_internal.h"
#include "pages_book.h"

namespace asl {

namespace {

constexpr int kFillThreads = 256;
constexpr int kPlanTokens = 8192;          // tokens that the bookkeeping workgroup fills in itself; more take a launch of their own

// What is known of a request when its tokens are filled in.
struct Placed {
  int row, old;            // -1: out of range
  bool fits;               // its row has grown
};

// Token k of a request whose row is `row`: slot and position.  depth: how far it stands behind the row's old tokens in the sequence.
__device__ __forceinline__ bool place_token(const PlanArgs& a, const Placed& p, int k, int depth, int64_t* slot, int* pos) {
  *slot = -1;
  *pos = -1;
  if (p.row < 0) return true;
  *pos = (int)((uint32_t)(p.old + depth) + (uint32_t)(a.pruned != nullptr ? a.pruned[p.row] : 0));
  if (!p.fits) return true;
  const int at = p.old + k;
  const int page = a.table[(int64_t)p.row * a.map.row_stride + (at >> a.map.ps_shift)];
  if ((uint32_t)page >= (uint32_t)a.map.n_pages) return false;
  *slot = (int64_t)page * a.map.ps + (at & (a.map.ps - 1));
  return true;
}

struct PlanLds {
  BookLds book;
  unsigned long long wave[kBookThreads / 64];
  uint32_t room;                           // tokens ahead of the first request that does not fit
  int32_t cu[kPagedMaxSeqs + 1];
  int32_t row[kPagedMaxSeqs], old[kPagedMaxSeqs];
  int16_t parent[kPlanTokens];
};

// Inclusive prefix sum over the workgroup of numbers whose sum may pass 32 bits; *total gets the sum.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long x, PlanLds& l, unsigned long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const unsigned long long y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  __syncthreads();                         // the last reader of l.wave is done
  if (lane == 63) l.wave[wave] = x;
  __syncthreads();
  unsigned long long before = 0, all = 0;
  for (int w = 0; w < kBookThreads / 64; ++w) {
    const unsigned long long s = l.wave[w];
    before += w < wave ? s : 0;
    all += s;
  }
  *total = all;
  return before + x;
}

// The requests' pages, where their tokens begin, and (FILL) each token's slot and position: one workgroup, bound by the latency of loads
// that depend on each other (requests, lengths, counts, pages).  A draft's parents are taken to LDS, where a node's depth is a walk.
// 64 drafts of 5 to 32 nodes 13 to 15 us, 24 prompts 8 to 10 and 3 to 4 for the launch that fills in their tokens.
template <bool FILL>
__global__ void __launch_bounds__(kBookThreads) pages_plan_kernel(PlanArgs a) {
  __shared__ PlanLds l;
  const PageMap& m = a.map;
  Growth g[kBookUnroll];
  int row[kBookUnroll], add[kBookUnroll];
  unsigned long long upto[kBookUnroll];
  if (threadIdx.x == 0) l.room = (uint32_t)a.total;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    row[u] = i < a.n ? a.rows[i] : -1;
    add[u] = i < a.n ? a.add[i] : 0;
    if (add[u] < 0) bad = true;
  }
  unsigned long long base = 0;
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
    upto[u] = 0;
    if (u * kBookThreads >= a.n) break;
    unsigned long long total;
    upto[u] = base + block_scan((unsigned long long)max(add[u], 0), l, &total);
    base += total;
    const unsigned long long from = upto[u] - (unsigned long long)max(add[u], 0);
    if (upto[u] > (unsigned long long)a.total && from <= (unsigned long long)a.total) {
      atomicMin(&l.room, (uint32_t)from);
      bad = true;
    }
  }
  __syncthreads();
  const uint32_t room = l.room;
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i >= a.n) continue;
    const int end = (int)(upto[u] < room ? (uint32_t)upto[u] : room);
    a.cu[i + 1] = end;
    if (FILL) l.cu[i + 1] = end;
    // (a request that does not fit in the tokens that there is room for is left out like one that is out of range)
    const bool too_long = a.parent != nullptr && add[u] > kPlanNodes;
    if (upto[u] > room || too_long || !g[u].take(m, a.kv_len, row[u], add[u])) bad = true;
  }
  if (threadIdx.x == 0) {
    a.cu[0] = 0;
    if (FILL) l.cu[0] = 0;
  }
  const int got = give_pages(m, a.table, a.kv_len, a.refs, a.rows, a.n, a.fresh, g, l.book);
#pragma unroll
  for (int u = 0; u < kBookUnroll; ++u) {
    const int i = u * kBookThreads + (int)threadIdx.x;
    if (i >= a.n) continue;
    if (FILL) {
      l.row[i] = g[u].row;
      l.old[i] = g[u].len;
    } else {
      a.placed[i] = make_int4(g[u].row, g[u].len, l.book.incl[i] <= got ? 1 : 0, 0);
    }
  }
  __syncthreads();
  if (FILL) {
    if (a.parent != nullptr) {
      for (int j = threadIdx.x; j < a.total; j += kBookThreads) {
        const int i = sequence_of(l.cu, a.n, j), p = a.parent[j];
        if (i >= a.n || j >= l.cu[i + 1]) continue;
        const bool in = p >= -1 && p < j - l.cu[i];
        bad = bad || !in;
        l.parent[j] = (int16_t)(in ? p : -1);
      }
      __syncthreads();
    }
    for (int j = threadIdx.x; j < a.total; j += kBookThreads) {
      const int i = sequence_of(l.cu, a.n, j), c0 = l.cu[i];
      const bool in = i < a.n && j < l.cu[i + 1];
      const Placed p = {in ? l.row[i] : -1, l.old[i], l.book.incl[i] <= got};
      int depth = j - c0;
      if (a.parent != nullptr && in) {
        int k = depth;
        depth = -1;
        for (; k >= 0; k = l.parent[c0 + k]) ++depth;
      }
      int64_t slot;
      int pos;
      if (!place_token(a, p, j - c0, depth, &slot, &pos)) bad = true;
      a.slot[j] = slot;
      a.pos[j] = pos;
    }
  }
  if (bad) paged_fault(m);
}

// The tokens of larger plans: a thread each.
__global__ void __launch_bounds__(kFillThreads) pages_plan_fill_kernel(PlanArgs a) {
  extern __shared__ int32_t cu[];          // [n + 1]
  for (int i = threadIdx.x; i <= a.n; i += kFillThreads) cu[i] = a.cu[i];
  __syncthreads();
  const int j = (int)(blockIdx.x * kFillThreads + threadIdx.x);
  if (j >= a.total) return;
  const int i = sequence_of(cu, a.n, j), c0 = cu[i];
  const bool in = i < a.n && j < cu[i + 1];
  const int4 f = a.placed[i];
  bool bad = false;
  int depth = j - c0;
  if (a.parent != nullptr && in && f.x >= 0) {
    int k = depth;                         // (less than kPlanNodes, or the request is out of range)
    depth = -1;
    while (k >= 0) {                       // (a parent stands before its node: the walk ends)
      ++depth;
      const int p = a.parent[c0 + k];
      if (p < -1 || p >= k) {
        bad = true;
        break;
      }
      k = p;
    }
  }
  const Placed p = {in ? f.x : -1, f.y, f.z != 0};
  int64_t slot;
  int pos;
  if (!place_token(a, p, j - c0, depth, &slot, &pos)) bad = true;
  a.slot[j] = slot;
  a.pos[j] = pos;
  if (bad) paged_fault(a.map);
}

// ---------------------------------------------------------------------------------------------------------------------
typedef uint32_t Piece __attribute__((ext_vector_type(4)));              // 16 bytes

constexpr int kAcceptThreads = 256;
constexpr int kAcceptUnroll = 4;           // pieces that a thread has on their way

// Node path[t] of a draft becomes the draft's token t, t < a.  The path ascends, so path[t] >= t: pieces are taken in the order of t, some at
// a time, all read before the first of them is written, and none that is still to be read is written to.
// grid: x = sequences, y = slices (layer, K or V).  The workgroup that is the last of its sequence to have copied changes the row's length,
// which all of them read, and gives the pages behind it back.  Bound by loads that depend on each other: 64 rows of 8 layers, 6.4 MB, 9.8 us,
// 3 rows of two 5.1; several slices a workgroup were slower, since a chain is then walked more than once.
__global__ void __launch_bounds__(kAcceptThreads) pages_accept_kernel(AcceptArgs a) {
  __shared__ int64_t from[kTreeNodes], to[kTreeNodes];
  __shared__ int32_t node[kTreeNodes];
  __shared__ int32_t end, first, last;
  const PageMap& m = a.map;
  const int b = (int)blockIdx.x, tid = (int)threadIdx.x;
  const int r = a.rows[b], c0 = a.cu[b], c1 = a.cu[b + 1], wanted = a.n_path[b];
  int len;
  bool bad = !row_length(m, r, &len) || c0 < 0 || c1 < c0 || wanted < 0 || wanted > a.path_stride || wanted > c1 - c0 ||
             (a.slot != nullptr && c1 > a.total);
  // a row that did not get its pages has no draft: its last tokens are others
  const bool drafted = bad || a.slot == nullptr || c1 == c0 || a.slot[c0] >= 0;
  if (drafted && c1 - c0 > len) bad = true;
  const bool sound = !bad && drafted;
  const int base = len - (c1 - c0), n = sound ? wanted : 0;
  if (tid == 0) {
    end = n;
    first = n;
  }
  for (int t = tid; t < n; t += kAcceptThreads) node[t] = a.path[(int64_t)b * a.path_stride + t];
  __syncthreads();
  for (int t = tid; t < n; t += kAcceptThreads) {
    // (the first entry that does not ascend ends the path)
    const int x = node[t];
    if (x < 0 || x >= c1 - c0 || (t > 0 && x <= node[t - 1])) {
      atomicMin(&end, t);
      bad = true;
    }
    if (x != t) atomicMin(&first, t);
  }
  __syncthreads();
  const int keep = end, t0 = min(first, keep);             // those ahead of t0 stand where they belong
  if (a.n_layers > 0) {
    for (int t = t0 + tid; t < keep; t += kAcceptThreads) {
      from[t] = token_offset(m, r, base + node[t]);
      to[t] = token_offset(m, r, base + t);
      if (from[t] < 0 || to[t] < 0) {
        bad = true;
        to[t] = -1;
      }
    }
    __syncthreads();
    const int slice = (int)blockIdx.y;
    char* pages = (char*)((slice & 1) == 0 ? a.k_ptrs[slice >> 1] : a.v_ptrs[slice >> 1]);
    const uint32_t per = (uint32_t)a.Hk * (uint32_t)a.cpr, total = (uint32_t)(keep - t0) * per;
    for (uint32_t q0 = 0; q0 < total; q0 += kAcceptThreads * kAcceptUnroll) {
      Piece x[kAcceptUnroll];
      int64_t dst[kAcceptUnroll];
#pragma unroll
      for (int u = 0; u < kAcceptUnroll; ++u) {
        const uint32_t q = q0 + (uint32_t)(u * kAcceptThreads + tid);
        dst[u] = -1;
        if (q >= total) continue;
        const uint32_t t = q / per, e = q - t * per, h = a.cpr_shift >= 0 ? e >> a.cpr_shift : e / (uint32_t)a.cpr;
        if (to[t0 + t] < 0) continue;
        const int64_t within = (int64_t)h * m.head + (int64_t)(e - h * (uint32_t)a.cpr) * 16;
        dst[u] = to[t0 + t] + within;
        x[u] = *(const Piece*)(pages + from[t0 + t] + within);
      }
      __builtin_amdgcn_s_waitcnt(0);       // the pieces are there, those of the other wavefronts after the barrier
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kAcceptUnroll; ++u)
        if (dst[u] >= 0) *(Piece*)(pages + dst[u]) = x[u];
    }
  }
  if (bad) paged_fault(m);
  if (tid == 0) {
    last = 0;
    if (__hip_atomic_fetch_add(&a.arrived[b], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == gridDim.y) {
      __hip_atomic_store(&a.arrived[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // (a row that another entry has changed meanwhile stays as that left it)
      last = sound && atomicCAS(&a.kv_len[r], len, base + keep) == len ? 1 : 0;
      if (drafted && last == 0) paged_fault(m);
    }
  }
  __syncthreads();
  if (last == 0) return;
  bad = false;
  for (int t = ((base + keep + m.ps - 1) >> m.ps_shift) + tid; t < (len + m.ps - 1) >> m.ps_shift; t += kAcceptThreads) {
    const int page = m.table[(int64_t)r * m.row_stride + t];
    if ((uint32_t)page >= (uint32_t)m.n_pages) {
      bad = true;
    } else if (atomicSub(&a.refs[page], 1) <= 0) {         // nobody held it
      atomicAdd(&a.refs[page], 1);
      bad = true;
    }
  }
  if (bad) paged_fault(m);
}

}  // namespace

hipError_t launch_pages_plan(const PlanArgs& a, hipStream_t st) {
  if (a.total <= kPlanTokens) {
    hipLaunchKernelGGL(pages_plan_kernel<true>, dim3(1), dim3(kBookThreads), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(pages_plan_kernel<false>, dim3(1), dim3(kBookThreads), 0, st, a);
  hipLaunchKernelGGL(pages_plan_fill_kernel, dim3((unsigned)(((int64_t)a.total + kFillThreads - 1) / kFillThreads)), dim3(kFillThreads),
                     (size_t)(a.n + 1) * sizeof(int32_t), st, a);
  return hipGetLastError();
}

hipError_t launch_pages_accept(const AcceptArgs& a, hipStream_t st) {
  if (a.n == 0) return hipSuccess;
  hipLaunchKernelGGL(pages_accept_kernel, dim3((unsigned)a.n, (unsigned)(a.n_layers > 0 ? 2 * a.n_layers : 1)), dim3(kAcceptThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace asl
