// Launches of one operand type's variants.
#pragma once

#include <algorithm>

#include "gc_linear_few.h"
#include "gc_linear_plan.h"
#include "gc_linear_tiles.h"

namespace gc {

// Tiles of a launch, at most (times the parts of the inner dimension they fit an int).
constexpr int64_t kMostTiles = 1 << 20;

template <class C>
void launch_tiles(LinearArgs p, hipStream_t stream) {
  const int64_t tiles_w = (p.n_out + C::kOut - 1) / C::kOut, most = std::max<int64_t>(1, kMostTiles / tiles_w) * C::kX;
  const int64_t n = p.n_rows, width = (p.gated ? 2 : 1) * (int64_t)p.partial_cols;
  for (int64_t r = 0; r < n; r += most) {
    p.n_rows = std::min(n - r, most);
    const int64_t tiles_x = (p.n_rows + C::kX - 1) / C::kX;
    k_linear_tiles<C><<<(unsigned)(tiles_x * tiles_w * p.parts), C::kThreads, 0, stream>>>(p, (int)tiles_x, (int)tiles_w);
    p.x += most * p.x_row;
    if (p.x_scale) p.x_scale += most;
    if (p.residual) p.residual += most * p.residual_row;
    if (p.partial) p.partial += most * width;
    p.out += most * p.out_row;
  }
}

template <class Few, bool kGated>
void launch_few(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  const dim3 grid((unsigned)((p.n_out + 15) / 16), (unsigned)p.parts);
  if constexpr (!kGated)
    if (plan.wide) return k_linear_few<Few, 8, false, true><<<dim3((unsigned)((p.n_out + 31) / 32)), 512, 0, stream>>>(p);
  if (plan.waves == 8) k_linear_few<Few, 8, kGated, false><<<grid, 512, 0, stream>>>(p);
  else k_linear_few<Few, 16, kGated, false><<<grid, 1024, 0, stream>>>(p);
}

// Few: the operand type of few rows; Op: of tiles; kLargeX: rows of x of a wave of the largest tiles.  Tiles of 128 hold two
// steps in LDS, and a compute unit two of them, or four where there are no two tiles for a unit (2411 x 1024 x 2736 bfloat16
// 39 us and 30; 2411 x 2736 gated x 1024 39 and 47).
template <class Few, class Op, int kLargeX, bool kGated>
void launch_kind(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  switch (plan.kind) {
    case kLinearFew: launch_few<Few, kGated>(p, plan, stream); break;
    case kLinearTiles32x64:
      if constexpr (Op::kTotals && !kGated) launch_tiles<Tiles<Op, 2, 2, 16, 32, 3, false>>(p, stream);
      break;
    case kLinearTiles64: launch_tiles<Tiles<Op, 2, 2, 32, 64, 3, kGated>>(p, stream); break;
    case kLinearTiles128: launch_tiles<Tiles<Op, 4, 2, 32, 64, 2, kGated>>(p, stream); break;
    case kLinearTiles128Deep: launch_tiles<Tiles<Op, 4, 2, 32, 64, 4, kGated>>(p, stream); break;
    case kLinearTiles192:
      if constexpr (!Op::kTotals) launch_tiles<Tiles<Op, 2, 4, 96, 64, 2, kGated>>(p, stream);
      break;
    default: launch_tiles<Tiles<Op, 2, 4, kLargeX, 64, 2, kGated>>(p, stream); break;
  }
}

template <class Few, class Op, int kLargeX>
void launch_linear(const LinearArgs& p, const LinearPlan& plan, hipStream_t stream) {
  if (p.gated) launch_kind<Few, Op, kLargeX, true>(p, plan, stream);
  else launch_kind<Few, Op, kLargeX, false>(p, plan, stream);
}

}  // namespace gc
