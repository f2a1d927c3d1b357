// Attention over a paged cache (attend_body.h): which kernels a call takes.  The kernels of bf16 with d <= 64 and of d <= 128 are compiled
// apart, in attend_64.hip and attend_128.hip.
#include "attend_body.h"

namespace asl {

hipError_t launch_attend(const PagedWorkspace& ws, const AttendArgs& a, int dtype, hipStream_t st) {
  if (a.total_q == 0 || a.n_seqs == 0) return hipSuccess;
  if (dtype == ASL_BF16) {
    if (a.d <= 64) return launch_attend_bf16_64(ws, a, st);
    if (a.d <= 128) return launch_attend_bf16_128(ws, a, st);
    return launch_d<__bf16, 256>(ws, a, st);
  }
  if (a.d <= 64) return launch_d<float, 64>(ws, a, st);
  if (a.d <= 128) return launch_d<float, 128>(ws, a, st);
  return launch_d<float, 256>(ws, a, st);
}

}  // namespace asl
