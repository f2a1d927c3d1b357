// The kernels of attend_body.h for drafted trees, bf16 and d <= 64.
#include "attend_steps.h"

namespace asl {

hipError_t launch_attend_tree_bf16_64(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st) { return launch_d<__bf16, 64, true>(ws, a, st); }

}  // namespace asl
