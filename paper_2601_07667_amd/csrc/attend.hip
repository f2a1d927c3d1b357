// Attention over a paged cache: for query i of a sequence of n_q queries and L keys, over the keys j < lim_i,
//   x_j = scale q_i . k_j,  m = max x_j,  z = sum exp(x_j - m),  out = sum exp(x_j - m) v_j / z,  lse = m + log z,
// lim_i = L - n_q + i + 1 (causal: the queries are the sequence's last tokens) or L.  A row without keys gets out 0, lse -inf.
#include "paged.h"

#include "asl_internal.h"

namespace asl {

namespace {

constexpr int kSimpleThreads = 256;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__bf16 x) { return (float)x; }

// One workgroup per query token and head, 256 keys at a time: a key's logit per thread, then an output dimension per thread.
template <typename T>
__global__ void __launch_bounds__(kSimpleThreads) attend_simple_kernel(AttendArgs a) {
  __shared__ float qs[kPagedMaxDim], ps[kSimpleThreads], red[4];
  __shared__ int64_t off[kSimpleThreads];
  const int tok = blockIdx.x, hq = blockIdx.y, hk = hq / a.G, tid = threadIdx.x;
  int lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu_q[mid] <= tok) lo = mid; else hi = mid;
  }
  const PageMap& m = a.map;
  const int row = a.rows != nullptr ? a.rows[lo] : lo;
  int lim = 0;
  if ((uint32_t)row < (uint32_t)m.n_rows && a.cu_q[lo] <= tok && tok < a.cu_q[lo + 1]) {
    const int64_t cap = (int64_t)m.row_stride * m.ps;
    const int L = m.kv_len[row];
    if (L < 0 || L > cap) { if (tid == 0) atomicOr(m.fault, kFaultPaged); }
    else lim = a.causal ? max(0, L - (a.cu_q[lo + 1] - tok) + 1) : L;
  } else if (tid == 0) {
    atomicOr(m.fault, kFaultPaged);
  }
  const T* q = (const T*)a.q + (int64_t)tok * a.qt + (int64_t)hq * a.qh;
  for (int e = tid; e < a.d; e += kSimpleThreads) qs[e] = to_f(q[e]);
  __syncthreads();
  float mx = -INFINITY, z = 0.f, acc = 0.f;
  for (int j0 = 0; j0 < lim; j0 += kSimpleThreads) {
    const int j = j0 + tid;
    float x = -INFINITY;
    int64_t o = -1;
    if (j < lim) {
      const int page = m.table[(int64_t)row * m.row_stride + (j >> m.ps_shift)];
      if ((uint32_t)page < (uint32_t)m.n_pages) {
        o = (int64_t)page * m.page + (int64_t)(j & (m.ps - 1)) * m.tok + (int64_t)hk * m.head;
        const T* k = (const T*)((const char*)a.k + o);
        float s = 0.f;
        for (int e = 0; e < a.d; ++e) s += qs[e] * to_f(k[e]);
        x = s * a.scale;
      } else {
        atomicOr(m.fault, kFaultPaged);
      }
    }
    float w = x;
    for (int o2 = 32; o2 > 0; o2 >>= 1) w = fmaxf(w, __shfl_xor(w, o2));
    if ((tid & 63) == 0) red[tid >> 6] = w;
    __syncthreads();
    const float top = fmaxf(mx, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float base = top == -INFINITY ? 0.f : top;
    const float p = o >= 0 ? expf(x - base) : 0.f, shrink = expf(mx - base);
    ps[tid] = p;
    off[tid] = o;
    float sum = p;
    for (int o2 = 32; o2 > 0; o2 >>= 1) sum += __shfl_xor(sum, o2);
    __syncthreads();                                       // red has been read
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    z = z * shrink + (red[0] + red[1]) + (red[2] + red[3]);
    acc *= shrink;
    mx = top;
    if (tid < a.d)
      for (int t = 0; t < kSimpleThreads; ++t)
        if (off[t] >= 0) acc += ps[t] * to_f(((const T*)((const char*)a.v + off[t]))[tid]);
    __syncthreads();
  }
  if (tid < a.d) ((T*)a.out)[(int64_t)tok * a.ot + (int64_t)hq * a.oh + tid] = (T)(z == 0.f ? 0.f : acc / z);
  if (tid == 0 && a.lse != nullptr) a.lse[(int64_t)hq * a.total_q + tok] = z == 0.f ? -INFINITY : mx + logf(z);
}

}  // namespace

hipError_t launch_attend(const PagedWorkspace&, const AttendArgs& a, int dtype, hipStream_t st) {
  if (a.total_q == 0 || a.n_seqs == 0) return hipSuccess;
  const dim3 grid((unsigned)a.total_q, (unsigned)a.Hq);
  if (dtype == ASL_BF16)
    hipLaunchKernelGGL((attend_simple_kernel<__bf16>), grid, dim3(kSimpleThreads), 0, st, a);
  else
    hipLaunchKernelGGL((attend_simple_kernel<float>), grid, dim3(kSimpleThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace asl
