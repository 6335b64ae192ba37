// Matrix products of 8-bit operands.
#include "gc_linear_launch.h"

namespace gc {
void launch_linear_e4m3(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  if (p.out_f32) launch_linear<FewE4M3, E4M3Exact, 128>(p, plan, stream);
  else launch_linear<FewE4M3, E4M3, 128>(p, plan, stream);
}
}  // namespace gc
