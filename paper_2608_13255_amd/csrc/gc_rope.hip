// Rotary positions, and the per-head RMS norms of queries and keys with the
// rotation in the same pass.
//
// A column j of the rotation turns two channels (a, b) of a head to
// (a c - b s, b c + a s) with (c, s) = table[position][j].  One lane holds
// both channels of its columns (two runs of V channels), so nothing is
// exchanged for the turn; the norm's sum of squares is one butterfly over the
// lanes of a head.
//
// Memory-bound: each value is read and written once, about 3 operations a
// value (7 with the norm) against 4 or 8 bytes.  What counted: all of a
// wave's loads of heads issued before anything waits (the table's row and the norm's gains follow), the sixteen bytes of
// neighbouring lanes side by side, and arguments chosen between queries
// and keys in scalar registers.  196608 tokens x 32 heads x 128 bfloat16 with the
// norms: 538 us (6.0 TB/s of a copy's 6.5); 196608 x 16 x 128, 64 channels turned: 289 us
// (5.8 TB/s); 13823 x 16 x 64 float: 20.7 us (5.5 TB/s).  The table, in double: 4096 x 64 columns 5.2 us, 393216 x 64
// 107 us (1.9 TB/s written: bound by the sines and cosines), scaled 136.
#include <type_traits>

#include "gc_heads.h"

namespace gc {
namespace {

constexpr int kBlock = 256;
constexpr int64_t kOnceBytes = 64 << 20;   // read and written

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
  uint32_t head_groups;      // waves of a token
  float eps, inv_dim;
};

template <int kControl>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kControl, 0xf, 0xf, true));
}

// The sum over the 2^lanes_log2 lanes of a head, in every one of them.
// (Mirroring half a row, or a row, pairs lanes whose sums so far are of different parts.)
__device__ __forceinline__ float sum_lanes(float x, int lanes_log2) {
  if (lanes_log2 > 0) x += dpp<0xb1>(x);    // lane ^ 1
  if (lanes_log2 > 1) x += dpp<0x4e>(x);    // lane ^ 2
  if (lanes_log2 > 2) x += dpp<0x141>(x);   // half row mirrored
  if (lanes_log2 > 3) x += dpp<0x140>(x);   // row mirrored
  if (lanes_log2 > 4) x += __shfl_xor(x, 16);
  if (lanes_log2 > 5) x += __shfl_xor(x, 32);
  return x;
}

// 1 / sqrt(m): the hardware's estimate and one Newton step, and the divide
// and root where the estimate's range ends (0, tiny, infinite, NaN).
__device__ __forceinline__ float reciprocal_root(float m) {
  if (m > 0x1p-100f && m < 0x1p100f) {
    const float y = __builtin_amdgcn_rsqf(m);
    return __builtin_fmaf(0.5f * y, __builtin_fmaf(-m * y, y, 1.f), y);
  }
  return 1.f / __builtin_sqrtf(m);
}

// Keeps an argument in a scalar register: chosen between per lane, it would
// otherwise be loaded from the argument segment by each lane again.
template <class X>
__device__ __forceinline__ void in_register(X& x) {
  asm("" : "+s"(x));
}
// A device address as a pointer to device memory (not to any memory).
template <class X>
__device__ __forceinline__ X* at_address(uint64_t x) {
  return (X*)(__attribute__((address_space(1))) X*)x;
}

// One wave: 2^(6 - lanes_log2) heads kHeads times over, of one token or, where a
// token has fewer heads than that, of several.
template <class T, int V, int kHeads, bool kHalf, bool kNorm, bool kWhole, bool kOnce>
__global__ __launch_bounds__(kBlock) void k_rope(const RopeArgs p) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & ((1 << p.lanes_log2) - 1);
  const int slot = lane >> p.lanes_log2;
  const int tokens_log2 = 6 - p.lanes_log2 - p.slots_log2;
  const uint32_t set = wave / p.head_groups;   // of 2^tokens_log2 tokens
  const int64_t t = ((int64_t)set << tokens_log2) + (slot >> p.slots_log2);
  if (((int64_t)set << tokens_log2) >= p.n_tokens) return;
  const int h_first = (int)((wave - set * p.head_groups) << p.slots_log2) * kHeads + (slot & ((1 << p.slots_log2) - 1));
  const bool live = t < p.n_tokens && i * 2 * V < p.dim;
  // the lane's two runs of V channels, neighbouring lanes' side by side
  const int pair_lanes = p.half / V;
  const bool turns = i < pair_lanes;
  const int e0 = turns ? i * V : 2 * p.half + (i - pair_lanes) * V;
  const int e1 = e0 + (turns ? p.half : p.dim / 2 - p.half);

  // queries first, then keys
  const int total = p.heads[0] + p.heads[1];
  const auto head_of = [&](int u, const void* q, const void* k, int64_t q_token, int64_t k_token, int64_t q_head, int64_t k_head) {
    const int h = h_first + (u << p.slots_log2);
    uint64_t q_at = (uint64_t)q, k_at = (uint64_t)k;
    in_register(q_at), in_register(k_at), in_register(q_token), in_register(k_token), in_register(q_head), in_register(k_head);
    const bool key = h >= p.heads[0];
    return at_address<T>(key ? k_at : q_at) + t * (key ? k_token : q_token) + (key ? h - p.heads[0] : h) * (key ? k_head : q_head);
  };
  using Vec = HeadVec<T, V>;
  typename Vec::type raw[kHeads][2];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    raw[u][0] = raw[u][1] = 0;
    if (live && h_first + (u << p.slots_log2) < total) {   // on its way while the table's row is looked up
      const T* x = head_of(u, p.in[0], p.in[1], p.in_token[0], p.in_token[1], p.in_head[0], p.in_head[1]);
      raw[u][0] = load_vec<kOnce, typename Vec::type>(x + e0);
      raw[u][1] = load_vec<kOnce, typename Vec::type>(x + e1);
    }
  }

  float c[V], s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    c[j] = 1.f;
    s[j] = 0.f;
  }
  if (live && turns) {
    const int32_t* pos = p.positions + t * p.sec.n;
    // half pairs: columns i V ..; interleaved ones: those of both runs, V / 2 each
    constexpr int kRun = kHalf ? V : V / 2;
#pragma unroll
    for (int run = 0; run < V / kRun; ++run) {
      const int col = i * kRun + run * (p.half / 2);
      if constexpr (kWhole) {   // a run's columns belong to one axis
        int ax = 0;
        for (int k = 0; k + 1 < p.sec.n; ++k) ax += col >= p.sec.end[k];
        const int64_t at = pos[ax];
        if (at >= 0 && at < p.n_pos) {
          float w[2 * kRun];
          load_heads<2 * kRun>(p.table + (at * p.half + col) * 2, w);
#pragma unroll
          for (int j = 0; j < kRun; ++j) c[run * kRun + j] = w[2 * j], s[run * kRun + j] = w[2 * j + 1];
        } else {
#pragma unroll
          for (int j = 0; j < kRun; ++j) c[run * kRun + j] = s[run * kRun + j] = __builtin_nanf("");
        }
      } else {
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
          int ax = 0;
          for (int k = 0; k + 1 < p.sec.n; ++k) ax += col + j >= p.sec.end[k];
          const int64_t at = pos[ax];
          if (at >= 0 && at < p.n_pos) {
            float w[2];
            load_heads<2>(p.table + (at * p.half + col + j) * 2, w);
            c[run * kRun + j] = w[0], s[run * kRun + j] = w[1];
          } else {
            c[run * kRun + j] = s[run * kRun + j] = __builtin_nanf("");
          }
        }
      }
    }
  }

#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    float a[V], b[V];
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] = Vec::at(raw[u][0], j), b[j] = Vec::at(raw[u][1], j);
    if constexpr (kNorm) {
      float q = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) q = __builtin_fmaf(a[j], a[j], __builtin_fmaf(b[j], b[j], q));
      const float r = reciprocal_root(__builtin_fmaf(sum_lanes(q, p.lanes_log2), p.inv_dim, p.eps));
      if (live) {
        uint64_t q_gain = (uint64_t)p.gain[0], k_gain = (uint64_t)p.gain[1];
        in_register(q_gain), in_register(k_gain);
        const float* gain = at_address<float>(h_first + (u << p.slots_log2) >= p.heads[0] ? k_gain : q_gain);
        float g[V];
        load_heads<V>(gain + e0, g);
#pragma unroll
        for (int j = 0; j < V; ++j) a[j] = a[j] * r * g[j];
        load_heads<V>(gain + e1, g);
#pragma unroll
        for (int j = 0; j < V; ++j) b[j] = b[j] * r * g[j];
      }
    }
    if (turns) {
      if constexpr (kHalf) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float x = a[j], y = b[j];
          a[j] = __builtin_fmaf(x, c[j], -(y * s[j]));
          b[j] = __builtin_fmaf(y, c[j], x * s[j]);
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float& x = 2 * j < V ? a[2 * j] : b[2 * j - V];
          float& y = 2 * j < V ? a[2 * j + 1] : b[2 * j + 1 - V];
          const float x0 = x, y0 = y;
          x = __builtin_fmaf(x0, c[j], -(y0 * s[j]));
          y = __builtin_fmaf(y0, c[j], x0 * s[j]);
        }
      }
    }
    if (live && h_first + (u << p.slots_log2) < total) {
      T* y = head_of(u, p.out[0], p.out[1], p.out_token[0], p.out_token[1], p.out_head[0], p.out_head[1]);
      store_heads<V, kOnce>(y + e0, a);
      store_heads<V, kOnce>(y + e1, b);
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
  const int token_sets_log2 = 6 - p.lanes_log2 - p.slots_log2;
  const int64_t sets = (p.n_tokens + (1 << token_sets_log2) - 1) >> token_sets_log2;
  // Four times the heads a wave where that leaves each compute unit 32 waves (196608 x 32 x 128 bfloat16: 536 us against
  // 575, 5741 x 32 x 80 float: 25 against 27); else the shorter waves (1024 x 32 x 64: 5.9 us against 7.2).
  const auto groups = [&](int heads) { return (int64_t)((total + (heads << p.slots_log2) - 1) / (heads << p.slots_log2)); };
  const bool many = sets * groups(4) >= 32 * 256;
  p.head_groups = (uint32_t)groups(many ? 4 : 1);
  bool whole = true;
  const int run = layout == GC_ROPE_HALF ? V : V / 2;   // columns that a lane takes from one row
  for (int a = 0; a < p.sec.n; ++a) whole = whole && p.sec.end[a] % run == 0;
  if (layout != GC_ROPE_HALF) whole = whole && p.half / 2 % run == 0;
  // Past the caches what is over twice the L2 caches' 32 MiB (13823 x 16 x 64 float: 20.8 us against 23.0), if the lanes'
  // runs are whole lines of 128 bytes (runs of 64 bytes: 307 us past the caches, 287 through them).
  const int rest = p.dim / 2 - p.half;
  const bool once = 2 * p.n_tokens * total * p.dim * (int64_t)sizeof(T) >= kOnceBytes &&
                    p.half * (int)sizeof(T) % 128 == 0 && rest * (int)sizeof(T) % 128 == 0;
  const auto launch_one = [&](auto half, auto all, auto past, dim3 grid) {
    if (many)
      hipLaunchKernelGGL((k_rope<T, V, 4, decltype(half)::value, kNorm, decltype(all)::value, decltype(past)::value>), grid,
                         dim3(kBlock), 0, stream, p);
    else
      hipLaunchKernelGGL((k_rope<T, V, 1, decltype(half)::value, kNorm, decltype(all)::value, false>), grid, dim3(kBlock), 0,
                         stream, p);
  };
  // a launch's threads are counted in 32 bits: at most 2^25 waves at a time
  const int64_t most = ((int64_t)1 << 25) / p.head_groups << token_sets_log2, n_tokens = p.n_tokens;
  const auto go = [&](auto half, auto all, auto past) {
    for (int64_t done = 0; done < n_tokens; done += most) {
      p.n_tokens = n_tokens - done < most ? n_tokens - done : most;
      const int64_t waves = ((p.n_tokens + (1 << token_sets_log2) - 1) >> token_sets_log2) * p.head_groups;
      launch_one(half, all, past, dim3((unsigned)((waves + kBlock / 64 - 1) / (kBlock / 64))));
      p.positions += p.n_tokens * p.sec.n;
      for (int i = 0; i < 2; ++i) {
        if (p.heads[i] == 0) continue;
        p.in[i] = (const T*)p.in[i] + p.n_tokens * p.in_token[i];
        p.out[i] = (T*)p.out[i] + p.n_tokens * p.out_token[i];
      }
    }
  };
  const auto with = [&](auto half, auto all) { once ? go(half, all, std::true_type{}) : go(half, all, std::false_type{}); };
  const auto axes = [&](auto half) { whole ? with(half, std::true_type{}) : with(half, std::false_type{}); };
  layout == GC_ROPE_HALF ? axes(std::true_type{}) : axes(std::false_type{});
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
  // (an eps that float32 rounds to 0 would make NaN of heads of zeros, one that it rounds to infinity would make 0 of all)
  if (!(eps >= 0.0) || !__builtin_isfinite((float)eps) || (eps > 0.0 && (float)eps == 0.f))
    return fail(GC_ERR_ARG, "%s: eps=%g must be finite and not negative, and as a float32 neither infinite nor 0 unless it is 0", who, eps);
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
