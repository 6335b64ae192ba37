// Matrix products with what follows them.
//
//   p = x_scale_i w_scale_j sum_k x_ik w_jk + bias_j,  out = act(p) (* p of the value rows) + residual
#include <algorithm>

#include "gc_linear_tiles.h"

namespace gc {
namespace {

// Tiles of a launch, at most (times the parts of the inner dimension they fit an int).
constexpr int64_t kMostTiles = 1 << 20;

constexpr int kCus = 256;

template <class C>
void launch_tiles(LinearArgs p, hipStream_t stream) {
  const int64_t tiles_w = (p.n_out + C::kOut - 1) / C::kOut, most = std::max<int64_t>(1, kMostTiles / tiles_w) * C::kX;
  const int64_t n = p.n_rows, width = (p.gated ? 2 : 1) * (int64_t)p.partial_cols;
  for (int64_t r = 0; r < n; r += most) {
    p.n_rows = std::min(n - r, most);
    const int64_t tiles_x = (p.n_rows + C::kX - 1) / C::kX;
    const int64_t blocks = tiles_x * tiles_w * p.parts;
    k_linear_tiles<C><<<(unsigned)blocks, C::kThreads, 0, stream>>>(p, (int)tiles_x, (int)tiles_w);
    p.x += most * p.x_row;
    if (p.x_scale) p.x_scale += most;
    if (p.residual) p.residual += most * p.residual_row;
    if (p.partial) p.partial += most * width;
    p.out += most * p.out_row;
  }
}

template <class Op>
void launch_linear(const LinearArgs& p, hipStream_t stream) {
  if (p.gated) launch_tiles<Tiles<Op, 2, 4, 128, 64, true>>(p, stream);
  else launch_tiles<Tiles<Op, 2, 4, 128, 64, false>>(p, stream);
}
template <>
void launch_linear<F32>(const LinearArgs& p, hipStream_t stream) {
  if (p.gated) launch_tiles<Tiles<F32, 2, 4, 64, 64, true>>(p, stream);
  else launch_tiles<Tiles<F32, 2, 4, 64, 64, false>>(p, stream);
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
  (void)gated;
  return 0;
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
  const int64_t need = gc_linear_workspace_bytes(n_rows, n_out, n_in, dtype, gated);
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
  p.parts = 1, p.part_bytes = (p.row_bytes + kStepBytes - 1) / kStepBytes * kStepBytes;
  if (dtype == GC_F32) launch_linear<F32>(p, stream);
  else if (dtype == GC_BF16) launch_linear<BF16>(p, stream);
  else if (p.out_f32) launch_linear<E4M3Exact>(p, stream);
  else launch_linear<E4M3>(p, stream);
  return after_launch(stream, who);
}
