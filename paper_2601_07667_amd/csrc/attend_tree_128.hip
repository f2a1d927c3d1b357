// The kernels of attend_body.h for drafted trees, bf16 and d <= 128.
#include "attend_steps.h"

namespace asl {

hipError_t launch_attend_tree_bf16_128(const PagedWorkspace& ws, const AttendArgs& a, hipStream_t st) { return launch_d<__bf16, 128, true>(ws, a, st); }

}  // namespace asl
