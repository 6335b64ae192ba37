// Matrix products with what follows them.
//
//   p = x_scale_i w_scale_j sum_k x_ik w_jk + bias_j,  out = act(p) (* p of the value rows) + residual
//
// A call cannot do without 2 n_rows n_in operations a weight row, and reading x and w and writing out once: few rows are bound by
// the weights' bytes, everything else by the matrix units.  Measured, us, with the time of the bound at a large
// product's 1570 (bfloat16), 2720 (8 bits) and 153 TFLOP/s (float32), or a large read's 7.0 TB/s:
//   1 x 6144 x 4096 bfloat16                                  11.9   7.2
//   16 x 8192 x 4096 in 8 bits                                 9.2   4.8
//   1024 x 1283 x 1024 float32, bias, GELU, residual          33.6  17.6
//   10403 x 2736 gated x 1024 bfloat16                         132    74
//   10403 x 1024 x 2736 bfloat16, bias, residual                68    37
//   24576 x 16384 x 4096 bfloat16, bias, GELU                 2490  2101
//   24576 x 8192 gated x 4096 in 8 bits                       1345  1213
#include <algorithm>
#include <cmath>

#include "gc_linear_plan.h"

namespace gc {
namespace {

// What a launch of tiles takes, in microseconds, from timings: a step with one tile on a compute unit, with two, and the
// rest of a tile.  Those of bfloat16 and of 8 bits were taken with an epilogue that was unrolled over all rows; in a loop it is
// faster (24576 x 16384 x 4096 bfloat16 2490 us, 2698 by these figures; 10403 x 2736 gated x 1024 129 and 142; 24576 x 8192 gated
// x 4096 in 8 bits 1340 and 1546).
struct TileCost {
  int kind, x, w;
  double one, two, rest;     // two = 0: a unit holds one
};
constexpr TileCost kCosts[] = {
    {kLinearTiles64, 64, 128, 0.42, 0.75, 1.5}, {kLinearTiles128, 128, 128, 0.45, 1.15, 2.5},
    {kLinearTiles192, 192, 256, 1.25, 0, 9},    {kLinearTiles256, 256, 256, 1.6, 0, 10}};
// (8 bits, two tiles of 128 on a unit: 2.0 is of the unrolled epilogue, which spilled 60 bytes a lane.  In a loop it spills none,
// and gated ones 36 of either type, so these sizes take larger tiles than they may need: 2048 x 4096 x 4096 tiles of 192, 52 us by
// these figures, where bfloat16's would have tiles of 128 take 39.  Neither gating nor a float32 result, whose products run at
// bfloat16's rate, is in the tables.)
constexpr TileCost kCostsE4M3[] = {
    {kLinearTiles64, 64, 128, 0.42, 0.8, 1.5}, {kLinearTiles128, 128, 128, 0.45, 2.0, 2.5},
    {kLinearTiles192, 192, 256, 1.35, 0, 9},   {kLinearTiles256, 256, 256, 1.7, 0, 10}};
// (float32: tiles of 32 x 64 where larger ones leave units idle; 1024 x 1283 x 1024 33.6 us, 44.5 in 336 tiles of 64 x 64)
constexpr TileCost kCostsF32[] = {
    {kLinearTiles32x64, 32, 64, 0.39, 0.66, 1.5},
    {kLinearTiles64, 64, 128, 1.2, 2.05, 1.5}, {kLinearTiles128, 128, 128, 2.05, 4.0, 2.5}, {kLinearTiles256, 128, 256, 3.75, 0, 4}};

struct CostList {
  const TileCost *first, *last;
  template <int kCount>
  explicit CostList(const TileCost (&c)[kCount]) : first(c), last(c + kCount) {}
  const TileCost* begin() const { return first; }
  const TileCost* end() const { return last; }
};
CostList costs_of(int dtype) { return dtype == GC_F32 ? CostList(kCostsF32) : dtype == GC_BF16 ? CostList(kCosts) : CostList(kCostsE4M3); }

// Variant and parts.  At most 16 rows: each weight is read once by one wave (1 x 6144 x 4096 bfloat16 12 us; in tiles with
// parts 16); a wave's share of a row where there are few weight rows is cut by more waves, then by parts (16 x 1024 gated x
// 2736 13 us whole, 9 in four; 1 x 16384 x 4096 in 8 bits 13.1, 14.3 and 16.6 with 8, 4 and 16 waves a block).  From 9 rows on
// a block reads as much of x as of 16 weight rows, so it takes 32 where enough blocks are left (16384 x 4096 bfloat16 with 16, 12, 8
// and 4 rows 30.0, 28.9, 28.6 and 28.2 us, with 16 weight rows 33.6, 30.9, 28.1 and 25.8).  Else the tiles, and the parts of the inner
// dimension, that take least: 4096^3 bfloat16 183, 137 and 104 us with tiles of 64, 128 and 256, 10403 x 1024 x 2736 81 with
// 256 and 69 with 192, 1024^3 10.6, 11.3 and 26, 128 x 1024 x 4096 28, 29 and 74 whole, 12.6 with 64 in eight parts.
constexpr int kWideRows = 9;
LinearPlan choose(int64_t n_rows, int n_out, int row_bytes, int dtype, int gated) {
  const int steps = (row_bytes + kStepBytes - 1) / kStepBytes;
  const auto in_parts = [&](int kind, int parts, int waves) {
    const int each = (steps + parts - 1) / parts;
    return LinearPlan{kind, (steps + each - 1) / each, each * kStepBytes, waves, false};
  };
  const double w_rows = gated ? 2.0 * n_out : n_out;
  if (n_rows <= kLinearFewRows) {
    const int blocks = (n_out + 15) / 16;
    const int parts = std::min({8, kCus / blocks, row_bytes / 1280});
    LinearPlan plan = in_parts(kLinearFew, std::max(1, parts), blocks <= kCus ? 16 : 8);
    plan.wide = !gated && n_rows >= kWideRows && blocks >= 2 * kCus;
    return plan;
  }
  LinearPlan best = {};
  double least = 0;
  for (const TileCost& c : costs_of(dtype)) {
    if (gated && c.kind == kLinearTiles32x64) continue;
    const double tiles = std::ceil((double)n_rows / c.x) * std::ceil(w_rows / c.w);
    for (const int parts : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (parts > 1 && (steps < 2 * parts || tiles * parts > 4 * kCus)) break;
      const LinearPlan plan = in_parts(c.kind, parts, 0);
      const double blocks = tiles * plan.parts, each = plan.part_bytes / kStepBytes, at_once = c.two > 0 ? 2 * kCus : kCus;
      const double rounds = std::floor(blocks / at_once), over = blocks - rounds * at_once;
      const double one = c.rest + each * c.one, two = c.two > 0 ? c.rest + each * c.two : one;
      double t = rounds * two + (over > kCus ? two : over > 0 ? one : 0);
      // the parts' sums out and back, and their launch
      if (plan.parts > 1) t += 3.5 + 8e-6 / 4 * plan.parts * (double)n_rows * w_rows;
      if (least > 0 && t >= least) continue;
      least = t, best = plan;
      if (c.kind == kLinearTiles128 && blocks <= kCus) best.kind = kLinearTiles128Deep;
    }
  }
  return best;
}

// Sums of the parts in their order, and the epilogue: eight columns a thread.  Memory-bound, and small beside what cutting a
// long inner dimension saves (128 x 1024 x 4096 bfloat16 12.6 us in eight parts, 28 whole).
template <bool kGated>
__global__ __launch_bounds__(256) void k_linear_join(const LinearArgs p, int64_t groups) {
  const int row_groups = p.partial_cols / 8;
  for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (int64_t)gridDim.x * 256) {
    const int64_t m = g / row_groups;
    const int n = (int)(g - m * row_groups) * 8;
    const float* from = p.partial + m * p.partial_cols * (kGated ? 2 : 1) + n;
    float a[8], b[8];
    load_heads<8>(from, a);
    if (kGated) load_heads<8>(from + p.partial_cols, b);
    for (int part = 1; part < p.parts; ++part) {
      float add[8];
      load_heads<8>(from + part * p.partial_part, add);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] += add[i];
      if (kGated) {
        load_heads<8>(from + part * p.partial_part + p.partial_cols, add);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] += add[i];
      }
    }
    if (p.whole && n + 8 <= p.n_out) {
      Columns c;
      RowAhead row;
      c.init<kGated>(p, n);
      row.load(p, m, n);
      finish<kGated>(p, c, m, row, a, b);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (n + i < p.n_out) {
          Column c;
          OneAhead row;
          c.init<kGated>(p, n + i);
          row.load(p, m, n + i);
          finish_one<kGated>(p, c, m, row, a[i], kGated ? b[i] : 0.f);
        }
    }
  }
}

int64_t workspace_bytes(const LinearPlan& plan, int64_t n_rows, int n_out, int gated) {
  return plan.parts > 1 ? plan.parts * n_rows * ((n_out + 7) / 8 * 8) * (gated ? 2 : 1) * (int64_t)sizeof(float) : 0;
}

constexpr int64_t kMostStride = (int64_t)1 << 40;
constexpr int kMostOut = 1 << 22;

int check_sizes(int64_t n_rows, int n_out, int n_in, int dtype, const char* who) {
  if (dtype != GC_F32 && dtype != GC_BF16 && dtype != GC_E4M3) return fail(GC_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
  if (n_rows < 0 || n_rows > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: n_rows=%lld outside [0, 2^31-1]", who, (long long)n_rows);
  if (n_out < 1 || n_out > kMostOut) return fail(GC_ERR_CAPACITY, "%s: n_out=%d outside [1, 2^22]", who, n_out);
  if (n_in < 1 || n_in > GC_MAX_INNER) return fail(GC_ERR_CAPACITY, "%s: n_in=%d outside [1, %d]", who, n_in, GC_MAX_INNER);
  if ((int64_t)n_in * row_type_bytes(dtype) % 16) return fail(GC_ERR_SHAPE, "%s: n_in=%d is not a whole number of 16 bytes", who, n_in);
  return GC_OK;
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" int64_t gc_linear_workspace_bytes(int64_t n_rows, int n_out, int n_in, int dtype, int gated) {
  clear_error();
  if (check_sizes(n_rows, n_out, n_in, dtype, "gc_linear_workspace_bytes")) return -1;
  return workspace_bytes(choose(n_rows, n_out, n_in * row_type_bytes(dtype), dtype, gated), n_rows, n_out, gated);
}

extern "C" int gc_linear(const gc_rows* x, const float* x_scale, const gc_rows* w, const float* w_scale, int64_t n_rows,
                         int n_out, int n_in, int dtype, const float* bias, int act, int gated, const gc_rows* residual,
                         const gc_rows* out, int out_dtype, void* workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  const char* who = "gc_linear";
  int rc = check_sizes(n_rows, n_out, n_in, dtype, who);
  if (rc) return rc;
  if (out_dtype != GC_F32 && (out_dtype != GC_BF16 || dtype == GC_F32))
    return fail(GC_ERR_DTYPE, "%s: out_dtype %d with dtype %d", who, out_dtype, dtype);
  if (act < GC_ACT_NONE || act > GC_ACT_GELU_TANH) return fail(GC_ERR_ARG, "%s: unknown activation %d", who, act);
  if (dtype != GC_E4M3 && (x_scale || w_scale)) return fail(GC_ERR_ARG, "%s: scales are given without 8-bit operands", who);
  if (n_rows == 0) return GC_OK;
  if ((rc = check_rows(x, dtype, true, GC_MAX_INNER, "x", who)) || (rc = check_rows(w, dtype, true, GC_MAX_INNER, "w", who)) ||
      (residual && (rc = check_rows(residual, out_dtype, false, kMostStride, "residual", who))) ||
      (rc = check_rows(out, out_dtype, false, kMostStride, "out", who)) || (rc = check_rows_out(*out, n_rows, n_out, "out", who)))
    return rc;
  if ((reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(w_scale) | reinterpret_cast<uintptr_t>(bias)) & 3)
    return fail(GC_ERR_ALIGN, "%s: x_scale, w_scale or bias misaligned", who);
  const LinearPlan plan = choose(n_rows, n_out, n_in * row_type_bytes(dtype), dtype, gated);
  const int64_t need = workspace_bytes(plan, n_rows, n_out, gated);
  if (need > 0 && !workspace) return fail(GC_ERR_ARG, "%s: workspace is null", who);
  if (ws_bytes < (size_t)need)
    return fail(GC_ERR_CAPACITY, "%s: workspace of %zu bytes is below the %lld required", who, ws_bytes, (long long)need);
  if (workspace && !aligned16(workspace)) return fail(GC_ERR_ALIGN, "%s: workspace misaligned", who);
  const int64_t es = row_type_bytes(dtype), eo = row_type_bytes(out_dtype), w_rows = gated ? 2 * (int64_t)n_out : n_out;
  const size_t xs_bytes = x_scale ? (size_t)n_rows * 4 : 0, ws_scale_bytes = w_scale ? (size_t)w_rows * 4 : 0, bias_bytes = bias ? (size_t)w_rows * 4 : 0;
  if (rows_overlap(*out, n_rows, n_out, eo, *x, n_rows, n_in, es)) return fail(GC_ERR_ALIAS, "%s: out overlaps x", who);
  if (rows_overlap(*out, n_rows, n_out, eo, *w, w_rows, n_in, es)) return fail(GC_ERR_ALIAS, "%s: out overlaps w", who);
  if (residual && rows_overlap(*out, n_rows, n_out, eo, *residual, n_rows, n_out, eo) && !same_rows(*out, n_rows, *residual, n_rows))
    return fail(GC_ERR_ALIAS, "%s: out overlaps residual", who);
  if (rows_overlap(*out, n_rows, n_out, eo, x_scale, xs_bytes) || rows_overlap(*out, n_rows, n_out, eo, w_scale, ws_scale_bytes) ||
      rows_overlap(*out, n_rows, n_out, eo, bias, bias_bytes))
    return fail(GC_ERR_ALIAS, "%s: out overlaps x_scale, w_scale or bias", who);
  if (need > 0) {
    const size_t nb = (size_t)need;
    if (rows_overlap(*out, n_rows, n_out, eo, workspace, nb) || rows_overlap(*x, n_rows, n_in, es, workspace, nb) ||
        rows_overlap(*w, w_rows, n_in, es, workspace, nb) || (residual && rows_overlap(*residual, n_rows, n_out, eo, workspace, nb)) ||
        overlaps(x_scale, xs_bytes, workspace, nb) || overlaps(w_scale, ws_scale_bytes, workspace, nb) || overlaps(bias, bias_bytes, workspace, nb))
      return fail(GC_ERR_ALIAS, "%s: workspace overlaps another argument", who);
  }
  LinearArgs p = {};
  p.x = (const char*)x->data, p.w = (const char*)w->data;
  p.x_row = n_rows > 1 ? x->stride * es : 0, p.w_row = w_rows > 1 ? w->stride * es : 0;
  p.x_scale = x_scale, p.w_scale = w_scale, p.bias = bias;
  if (residual) p.residual = (const char*)residual->data, p.residual_row = residual->stride * eo;
  p.out = (char*)out->data, p.out_row = out->stride * eo;
  p.n_rows = n_rows, p.n_out = n_out, p.row_bytes = (int)(n_in * es);
  p.act = act, p.gated = gated != 0, p.out_f32 = out_dtype == GC_F32;
  p.whole = rows_aligned(*out, n_rows, 16, (int)eo) && (!residual || rows_aligned(*residual, n_rows, 16, (int)eo));
  p.parts = plan.parts, p.part_bytes = plan.part_bytes;
  p.partial = reinterpret_cast<float*>(workspace);
  p.partial_cols = (n_out + 7) / 8 * 8, p.partial_part = n_rows * p.partial_cols * (gated ? 2 : 1);
  if (dtype == GC_F32) launch_linear_f32(p, plan, stream);
  else if (dtype == GC_BF16) launch_linear_bf16(p, plan, stream);
  else launch_linear_e4m3(p, plan, stream);
  if (plan.parts > 1) {
    const int64_t groups = n_rows * (p.partial_cols / 8);
    const unsigned blocks = (unsigned)std::min<int64_t>((groups + 255) / 256, 1 << 16);
    if (gated) k_linear_join<true><<<blocks, 256, 0, stream>>>(p, groups);
    else k_linear_join<false><<<blocks, 256, 0, stream>>>(p, groups);
  }
  return after_launch(stream, who);
}
