// Matrix products of bfloat16 operands.
#include "gc_linear_launch.h"

namespace gc {
void launch_linear_bf16(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  launch_linear<FewBF16, BF16, 128>(p, plan, stream);
}
}  // namespace gc
