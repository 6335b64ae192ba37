// How a matrix product is worked on: variant, and parts of the inner dimension.
#pragma once

#include "gc_linear.h"

namespace gc {

enum LinearKind : int {
  kLinearFew,       // at most 16 rows: each weight to the registers of one wave
  kLinearTiles32x64,  // 32 rows x 64 weight rows a block (float32, not gated)
  kLinearTiles64,   // 64 rows x 128 weight rows a block
  kLinearTiles128,  // 128 x 128, two of them on a compute unit
  kLinearTiles128Deep,  // one, with more steps on their way
  kLinearTiles192,  // 192 x 256 (bfloat16 and 8 bits)
  kLinearTiles256,  // 256 x 256 (float32: 128 x 256)
  kLinearKinds
};

struct LinearPlan {
  int kind, parts, part_bytes;
  int waves;      // of a block of kLinearFew
  bool wide;      // 32 weight rows a block of kLinearFew (not gated, one part)
};

constexpr int kLinearFewRows = 16;
constexpr int kCus = 256;

// one for each operand type (8 bits: by the result's type)
void launch_linear_f32(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream);
void launch_linear_bf16(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream);
void launch_linear_e4m3(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream);

}  // namespace gc
