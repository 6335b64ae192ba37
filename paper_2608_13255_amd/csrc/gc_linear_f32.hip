// Matrix products of float32 operands.
#include "gc_linear_launch.h"

namespace gc {
void launch_linear_f32(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  launch_linear<FewF32, F32, 64>(p, plan, stream);
}
}  // namespace gc
