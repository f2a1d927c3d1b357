// The kernels of attend_body.h for bf16 and d <= 128.
#include "attend_body.h"

namespace asl {

hipError_t launch_attend_bf16_128(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st) { return launch_d<__bf16, 128, false>(ws, a, st); }

}  // namespace asl
