// The kernels of attend_body.h for bf16 and d <= 64.
#include "attend_body.h"

namespace asl {

hipError_t launch_attend_bf16_64(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st) { return launch_d<__bf16, 64>(ws, a, st); }

}  // namespace asl
