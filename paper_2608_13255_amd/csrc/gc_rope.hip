// Rotary positions, and the per-head RMS norms of queries and keys with the
// rotation in the same pass.
//
// A column j of the rotation turns two channels (a, b) of a head to
// (a c - b s, b c + a s) with (c, s) = table[position][j].  One lane holds
// both channels of its columns (V columns: two accesses of V channels), so
// nothing is exchanged for the turn; the norm's sum of squares is one
// butterfly over the lanes of a head.
//
// Memory-bound: each value is read and written once, about 3 operations a
// value (7 with the norm) against 4 or 8 bytes.
#include "gc_heads.h"

namespace gc {
namespace {

constexpr int kBlock = 256;
constexpr int kUnroll = 4;   // heads a lane has in flight

struct Sections {
  int n;                     // axes
  int end[GC_MAX_AXES];      // first column past each axis
};

struct RopeArgs {
  const void* in[2];         // queries, keys
  void* out[2];
  int64_t in_token[2], in_head[2], out_token[2], out_head[2];   // strides, elements
  const float* gain[2];
  int heads[2];
  int64_t n_tokens, n_pos;
  const int32_t* positions;
  const float* table;
  Sections sec;
  int dim, half;             // half = R / 2 columns
  int lanes_log2;            // lanes of a head
  int slots_log2;            // heads of a token in a wave at a time
  float eps, inv_dim;
};

// One wave: 2^(6 - lanes_log2) heads at a time, of one token or, where a
// token has fewer heads than that, of several.
template <class T, int V, bool kHalf, bool kNorm, bool kWhole>
__global__ __launch_bounds__(kBlock) void k_rope(const RopeArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
  const int i = lane & ((1 << p.lanes_log2) - 1);
  const int slot = lane >> p.lanes_log2;
  const int tokens_log2 = 6 - p.lanes_log2 - p.slots_log2;
  const int64_t t = (wave << tokens_log2) + (slot >> p.slots_log2);
  const int h_first = slot & ((1 << p.slots_log2) - 1);
  if ((wave << tokens_log2) >= p.n_tokens) return;
  const bool live = t < p.n_tokens && i * 2 * V < p.dim;
  // the lane's two runs of V channels
  const bool turns = i * V < p.half;
  const int e0 = (turns && kHalf) ? i * V : 2 * i * V;
  const int e1 = (turns && kHalf) ? p.half + i * V : e0 + V;

  float c[V], s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    c[j] = 1.f;
    s[j] = 0.f;
  }
  if (live && turns) {
    const int32_t* pos = p.positions + t * p.sec.n;
    if constexpr (kWhole) {   // the lane's columns belong to one axis
      int ax = 0;
      for (int a = 0; a + 1 < p.sec.n; ++a) ax += i * V >= p.sec.end[a];
      const int64_t at = pos[ax];
      if (at >= 0 && at < p.n_pos) {
        const float* row = p.table + (at * p.half + i * V) * 2;
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          float w[4];
          load_heads<4>(row + 2 * j, w);
          c[j] = w[0], s[j] = w[1], c[j + 1] = w[2], s[j + 1] = w[3];
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) c[j] = s[j] = __builtin_nanf("");
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        int ax = 0;
        for (int a = 0; a + 1 < p.sec.n; ++a) ax += i * V + j >= p.sec.end[a];
        const int64_t at = pos[ax];
        if (at >= 0 && at < p.n_pos) {
          float w[2];
          load_heads<2>(p.table + (at * p.half + i * V + j) * 2, w);
          c[j] = w[0], s[j] = w[1];
        } else {
          c[j] = s[j] = __builtin_nanf("");
        }
      }
    }
  }

  const int total = p.heads[0] + p.heads[1];
  for (int h0 = h_first; h0 < total; h0 += kUnroll << p.slots_log2) {
    float a[kUnroll][V], b[kUnroll][V];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + (u << p.slots_log2);
#pragma unroll
      for (int j = 0; j < V; ++j) a[u][j] = b[u][j] = 0.f;
      if (live && h < total) {
        const int w = h >= p.heads[0];
        const T* x = (const T*)p.in[w] + t * p.in_token[w] + (int64_t)(h - (w ? p.heads[0] : 0)) * p.in_head[w];
        load_heads<V>(x + e0, a[u]);
        load_heads<V>(x + e1, b[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = h0 + (u << p.slots_log2);
      const int w = h >= p.heads[0];
      if constexpr (kNorm) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) q = __builtin_fmaf(a[u][j], a[u][j], __builtin_fmaf(b[u][j], b[u][j], q));
        for (int d = 1; d < (1 << p.lanes_log2); d <<= 1) q += __shfl_xor(q, d);
        const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(q, p.inv_dim, p.eps));
        if (live) {
          float g[V];
          load_heads<V>(p.gain[w] + e0, g);
#pragma unroll
          for (int j = 0; j < V; ++j) a[u][j] = a[u][j] * r * g[j];
          load_heads<V>(p.gain[w] + e1, g);
#pragma unroll
          for (int j = 0; j < V; ++j) b[u][j] = b[u][j] * r * g[j];
        }
      }
      if (live && h < total) {
        if (turns) {
          if constexpr (kHalf) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float x = a[u][j], y = b[u][j];
              a[u][j] = x * c[j] - y * s[j];
              b[u][j] = y * c[j] + x * s[j];
            }
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
              float& x = 2 * j < V ? a[u][2 * j] : b[u][2 * j - V];
              float& y = 2 * j < V ? a[u][2 * j + 1] : b[u][2 * j + 1 - V];
              const float u0 = x, u1 = y;
              x = u0 * c[j] - u1 * s[j];
              y = u1 * c[j] + u0 * s[j];
            }
          }
        }
        T* y = (T*)p.out[w] + t * p.out_token[w] + (int64_t)(h - (w ? p.heads[0] : 0)) * p.out_head[w];
        store_heads<V>(y + e0, a[u]);
        store_heads<V>(y + e1, b[u]);
      }
    }
  }
}

struct TableArgs {
  float* table;
  int64_t n;                 // entries
  int half;
  Sections sec;
  double log2_base;
  gc_rope_scaling sc;
  int scaled;
};

__global__ __launch_bounds__(kBlock) void k_rope_table(const TableArgs p) {
  for (int64_t e = (int64_t)blockIdx.x * kBlock + threadIdx.x; e < p.n; e += (int64_t)gridDim.x * kBlock) {
    const int64_t pos = e / p.half;
    const int j = (int)(e - pos * p.half);
    int ax = 0;
    for (int a = 0; a + 1 < p.sec.n; ++a) ax += j >= p.sec.end[a];
    const int begin = ax ? p.sec.end[ax - 1] : 0;
    double f = exp2(-p.log2_base * (double)(j - begin) / (double)(p.sec.end[ax] - begin));
    if (p.scaled) {
      const double r = p.sc.original_len * f / 6.283185307179586476925286766559;
      double g = r >= p.sc.low ? 1.0 : 0.0;
      if (p.sc.high > p.sc.low) g = fmin(1.0, fmax(0.0, (r - p.sc.low) / (p.sc.high - p.sc.low)));
      f = g * f + (1.0 - g) * f / p.sc.factor;
    }
    double sn, cs;
    sincos((double)pos * f, &sn, &cs);
    const double m = p.scaled ? p.sc.amplitude : 1.0;
    p.table[2 * e] = (float)(m * cs);
    p.table[2 * e + 1] = (float)(m * sn);
  }
}

int check_sections(const int32_t* sections, int n_axes, const char* who, Sections* out) {
  if (!sections) return fail(GC_ERR_ARG, "%s: sections is null", who);
  if (n_axes < 1 || n_axes > GC_MAX_AXES) return fail(GC_ERR_CAPACITY, "%s: n_axes=%d outside [1, %d]", who, n_axes, GC_MAX_AXES);
  out->n = n_axes;
  int sum = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 1 || sections[a] > GC_MAX_HEAD_DIM / 2)
      return fail(GC_ERR_SHAPE, "%s: sections[%d]=%d outside [1, %d]", who, a, sections[a], GC_MAX_HEAD_DIM / 2);
    sum += sections[a];
    out->end[a] = sum;
  }
  for (int a = n_axes; a < GC_MAX_AXES; ++a) out->end[a] = sum;
  if (sum % 2 || sum > GC_MAX_HEAD_DIM / 2)
    return fail(GC_ERR_SHAPE, "%s: the sections' sum %d is odd or above %d", who, sum, GC_MAX_HEAD_DIM / 2);
  return GC_OK;
}

// The checks the two calls share, and the lane layout.
int make_rope(RopeArgs* p, int64_t n_tokens, int dim, const int32_t* positions, const float* table, int64_t n_pos,
              const int32_t* sections, int n_axes, int layout, const char* who) {
  int rc = check_sections(sections, n_axes, who, &p->sec);
  if (rc) return rc;
  p->half = p->sec.end[n_axes - 1];
  if (2 * p->half > dim) return fail(GC_ERR_SHAPE, "%s: the sections turn %d channels of dim=%d", who, 2 * p->half, dim);
  if (layout != GC_ROPE_HALF && layout != GC_ROPE_INTERLEAVED) return fail(GC_ERR_ARG, "%s: unknown layout %d", who, layout);
  if (n_tokens < 0 || n_tokens > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: n_tokens=%lld outside [0, 2^31-1]", who, (long long)n_tokens);
  if (n_pos < 1 || n_pos > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: n_pos=%lld outside [1, 2^31-1]", who, (long long)n_pos);
  if (n_tokens > 0) {
    if (!positions || !table) return fail(GC_ERR_ARG, "%s: positions or table is null", who);
    if (!aligned16(table) || (reinterpret_cast<uintptr_t>(positions) & 3)) return fail(GC_ERR_ALIGN, "%s: table or positions misaligned", who);
  }
  p->n_tokens = n_tokens;
  p->n_pos = n_pos;
  p->positions = positions;
  p->table = table;
  p->dim = dim;
  return GC_OK;
}

template <class T, int V, bool kNorm>
void launch_v(RopeArgs& p, int layout, hipStream_t stream) {
  int lanes = 1;
  p.lanes_log2 = 0;
  while (lanes * 2 * V < p.dim) lanes *= 2, ++p.lanes_log2;
  const int total = p.heads[0] + p.heads[1];
  p.slots_log2 = 0;
  while ((1 << p.slots_log2) < total && (lanes << p.slots_log2) < 64) ++p.slots_log2;
  const int64_t per_block = (int64_t)(kBlock / 64) << (6 - p.lanes_log2 - p.slots_log2);
  const dim3 grid((unsigned)((p.n_tokens + per_block - 1) / per_block));
  bool whole = true;
  for (int a = 0; a < p.sec.n; ++a) whole = whole && p.sec.end[a] % V == 0;
  if (layout == GC_ROPE_HALF) {
    if (whole) hipLaunchKernelGGL((k_rope<T, V, true, kNorm, true>), grid, dim3(kBlock), 0, stream, p);
    else hipLaunchKernelGGL((k_rope<T, V, true, kNorm, false>), grid, dim3(kBlock), 0, stream, p);
  } else {
    if (whole) hipLaunchKernelGGL((k_rope<T, V, false, kNorm, true>), grid, dim3(kBlock), 0, stream, p);
    else hipLaunchKernelGGL((k_rope<T, V, false, kNorm, false>), grid, dim3(kBlock), 0, stream, p);
  }
}

// The widest access (16 bytes at most) of which both the turned pairs and the
// rest of the head are whole multiples.  R and dim are multiples of 4, so two
// channels always are.
template <class T, bool kNorm>
void launch(RopeArgs& p, int layout, hipStream_t stream) {
  const int rest = (p.dim - 2 * p.half) / 2;
  constexpr int most = 16 / (int)sizeof(T);
  if (most == 8 && p.half % 8 == 0 && rest % 8 == 0) launch_v<T, most, kNorm>(p, layout, stream);
  else if (p.half % 4 == 0 && rest % 4 == 0) launch_v<T, 4, kNorm>(p, layout, stream);
  else launch_v<T, 2, kNorm>(p, layout, stream);
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" int gc_rope_table(float* table, int64_t n_pos, const int32_t* sections, int n_axes, double base,
                             const gc_rope_scaling* scaling, hipStream_t stream) {
  clear_error();
  const char* who = "gc_rope_table";
  TableArgs p = {};
  int rc = check_sections(sections, n_axes, who, &p.sec);
  if (rc) return rc;
  if (!table) return fail(GC_ERR_ARG, "%s: table is null", who);
  if (!aligned16(table)) return fail(GC_ERR_ALIGN, "%s: table must be 16-byte aligned", who);
  if (n_pos < 1 || n_pos > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: n_pos=%lld outside [1, 2^31-1]", who, (long long)n_pos);
  if (!(base > 1.0) || !__builtin_isfinite(base)) return fail(GC_ERR_ARG, "%s: base must be finite and above 1", who);
  if (scaling) {
    if (!(scaling->factor > 0.0) || !__builtin_isfinite(scaling->factor) || !(scaling->original_len > 0.0) ||
        !__builtin_isfinite(scaling->original_len) || !(scaling->low <= scaling->high) || !__builtin_isfinite(scaling->amplitude))
      return fail(GC_ERR_ARG, "%s: scaling needs factor > 0, original_len > 0, low <= high and a finite amplitude", who);
    p.sc = *scaling;
    p.scaled = 1;
  }
  p.table = table;
  p.half = p.sec.end[n_axes - 1];
  p.n = n_pos * p.half;
  p.log2_base = __builtin_log2(base);
  const int64_t blocks = (p.n + kBlock - 1) / kBlock;
  hipLaunchKernelGGL(k_rope_table, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(kBlock), 0, stream, p);
  return after_launch(stream, who);
}

extern "C" int gc_rope(const gc_heads* x, int64_t n_tokens, int heads, int dim, int dtype, const int32_t* positions,
                       const float* table, int64_t n_pos, const int32_t* sections, int n_axes, int layout,
                       const gc_heads* out, hipStream_t stream) {
  clear_error();
  const char* who = "gc_rope";
  int rc = check_head_sizes(heads, dim, dtype, who);
  if (rc) return rc;
  RopeArgs p = {};
  rc = make_rope(&p, n_tokens, dim, positions, table, n_pos, sections, n_axes, layout, who);
  if (rc) return rc;
  if (n_tokens == 0) return GC_OK;
  if ((rc = check_heads(x, dtype, "x", who)) || (rc = check_heads(out, dtype, "out", who)) ||
      (rc = check_heads_out(*out, n_tokens, heads, dim, "out", who)))
    return rc;
  if (!same_heads(*x, *out) && heads_overlap(*x, n_tokens, heads, *out, n_tokens, heads, dim, dtype))
    return fail(GC_ERR_ALIAS, "%s: out overlaps x without being x", who);
  const size_t pos_bytes = (size_t)n_tokens * n_axes * 4, table_bytes = (size_t)n_pos * p.half * 8;
  const size_t out_bytes = (size_t)((n_tokens - 1) * out->token_stride + (heads - 1) * out->head_stride + dim) * dtype_bytes(dtype);
  if (overlaps(out->data, out_bytes, positions, pos_bytes) || overlaps(out->data, out_bytes, table, table_bytes))
    return fail(GC_ERR_ALIAS, "%s: out overlaps positions or table", who);
  p.in[0] = x->data, p.in_token[0] = x->token_stride, p.in_head[0] = x->head_stride;
  p.out[0] = out->data, p.out_token[0] = out->token_stride, p.out_head[0] = out->head_stride;
  p.heads[0] = heads;
  if (dtype == GC_F32) launch<float, false>(p, layout, stream);
  else launch<uint16_t, false>(p, layout, stream);
  return after_launch(stream, who);
}

extern "C" int gc_qk_norm_rope(const gc_heads* q, int heads, const gc_heads* k, int kv_heads, int64_t n_tokens, int dim,
                               int dtype, const float* q_gain, const float* k_gain, double eps, const int32_t* positions,
                               const float* table, int64_t n_pos, const int32_t* sections, int n_axes, int layout,
                               const gc_heads* q_out, const gc_heads* k_out, hipStream_t stream) {
  clear_error();
  const char* who = "gc_qk_norm_rope";
  int rc = check_head_sizes(heads, dim, dtype, who);
  if (rc) return rc;
  if ((rc = check_head_sizes(kv_heads, dim, dtype, who))) return rc;
  RopeArgs p = {};
  rc = make_rope(&p, n_tokens, dim, positions, table, n_pos, sections, n_axes, layout, who);
  if (rc) return rc;
  if (!(eps >= 0.0) || !__builtin_isfinite(eps)) return fail(GC_ERR_ARG, "%s: eps must be finite and not negative", who);
  if (n_tokens == 0) return GC_OK;
  if (!q_gain || !k_gain) return fail(GC_ERR_ARG, "%s: a gain is null", who);
  if (!aligned16(q_gain) || !aligned16(k_gain)) return fail(GC_ERR_ALIGN, "%s: gains must be 16-byte aligned", who);
  if ((rc = check_heads(q, dtype, "q", who)) || (rc = check_heads(k, dtype, "k", who)) ||
      (rc = check_heads(q_out, dtype, "q_out", who)) || (rc = check_heads(k_out, dtype, "k_out", who)) ||
      (rc = check_heads_out(*q_out, n_tokens, heads, dim, "q_out", who)) ||
      (rc = check_heads_out(*k_out, n_tokens, kv_heads, dim, "k_out", who)))
    return rc;
  const gc_heads* in[2] = {q, k};
  const gc_heads* out[2] = {q_out, k_out};
  const int n[2] = {heads, kv_heads};
  for (int o = 0; o < 2; ++o) {
    for (int i = 0; i < 2; ++i)
      if (!(o == i && same_heads(*in[i], *out[o])) && heads_overlap(*in[i], n_tokens, n[i], *out[o], n_tokens, n[o], dim, dtype))
        return fail(GC_ERR_ALIAS, "%s: %s overlaps %s", who, o ? "k_out" : "q_out", i ? "k" : "q");
    const size_t bytes = (size_t)((n_tokens - 1) * out[o]->token_stride + (n[o] - 1) * out[o]->head_stride + dim) * dtype_bytes(dtype);
    if (overlaps(out[o]->data, bytes, positions, (size_t)n_tokens * n_axes * 4) ||
        overlaps(out[o]->data, bytes, table, (size_t)n_pos * p.half * 8) || overlaps(out[o]->data, bytes, q_gain, (size_t)dim * 4) ||
        overlaps(out[o]->data, bytes, k_gain, (size_t)dim * 4))
      return fail(GC_ERR_ALIAS, "%s: an output overlaps positions, table or a gain", who);
  }
  if (heads_overlap(*q_out, n_tokens, heads, *k_out, n_tokens, kv_heads, dim, dtype))
    return fail(GC_ERR_ALIAS, "%s: q_out overlaps k_out", who);
  for (int i = 0; i < 2; ++i) {
    p.in[i] = in[i]->data, p.in_token[i] = in[i]->token_stride, p.in_head[i] = in[i]->head_stride;
    p.out[i] = out[i]->data, p.out_token[i] = out[i]->token_stride, p.out_head[i] = out[i]->head_stride;
    p.heads[i] = n[i];
    p.gain[i] = i ? k_gain : q_gain;
  }
  p.eps = (float)eps;
  p.inv_dim = 1.f / (float)dim;
  if (dtype == GC_F32) launch<float, true>(p, layout, stream);
  else launch<uint16_t, true>(p, layout, stream);
  return after_launch(stream, who);
}
