// Norms of the residual stream's sum, and rows in 8 bits with a scale each.
//
//   h = x + residual,  y = h / sqrt(mean h^2 + eps) * gain,
//   8 bits: scale = max |y| / 448,  q = y / scale
//
// Each value is read once and written once (twice with the sum), for about
// 6 operations: memory-bound.  A row lies in the registers of one wave or one
// block, so neither the mean nor the largest magnitude reads it again.  Measured, us, with
// the time of the bytes at a large copy's 6.5 TB/s:
//   196608 x 2048 bfloat16 with its sum, to 8 bits     470  434
//   16384 x 4096 float32 to 8 bits                      53   52
//   10403 x 4096 bfloat16 to 8 bits                     22   20
//   5741 x 1283 float32 with its sum                    21   18   (rows that begin anywhere)
//   1 x 4096 bfloat16                                  2.7        (a call from Python 8.1)
#include <cmath>

#include "gc_rows.h"

namespace gc {
namespace {

struct NormArgs {
  const void *x, *residual;
  void *total, *out;
  float* out_scale;
  const float* gain;
  int64_t x_row, residual_row, total_row, out_row;   // strides, elements
  int64_t n_rows;
  int width;
  int norm, eight;
  float eps, inv_width;
};

// 1 / sqrt(m): the hardware's estimate and one Newton step, and the divide
// and root where the estimate's range ends (0, tiny, infinite, NaN).
__device__ __forceinline__ float reciprocal_root_of(float m) {
  if (m > 0x1p-100f && m < 0x1p100f) {
    const float y = __builtin_amdgcn_rsqf(m);
    return __builtin_fmaf(0.5f * y, __builtin_fmaf(-m * y, y, 1.f), y);
  }
  return 1.f / __builtin_sqrtf(m);
}

// The sum, and the largest, over the lanes of a row (of a wave, if it has more), in every one of them.
template <int kLanes>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
  for (int i = 1; i < (kLanes < 64 ? kLanes : 64); i *= 2) x += __shfl_xor(x, i);
  return x;
}
template <int kLanes>
__device__ __forceinline__ uint32_t max_lanes(uint32_t x) {
#pragma unroll
  for (int i = 1; i < (kLanes < 64 ? kLanes : 64); i *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, i));
  return x;
}

// Groups of V values, 16 bytes in memory.  Where kWhole is not set they may begin anywhere and the last one may lie
// partly past the row's end (`have` values are in it): the hardware takes 16 bytes at any address.
template <class T, int V, bool kWhole, bool kOnce>
__device__ __forceinline__ void load_group(const T* p, int have, float (&x)[V]) {
  using Vec = typename HeadVec<T, V>::type;
  if (kWhole) {
    const Vec v = load_vec<kOnce, Vec>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = HeadVec<T, V>::at(v, i);
  } else if (have >= V) {
    Vec v;
    __builtin_memcpy(&v, p, sizeof(v));
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = HeadVec<T, V>::at(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = load_one(p + (i < have ? i : 0));
#pragma unroll
    for (int i = 1; i < V; ++i) x[i] = i < have ? x[i] : 0.f;
  }
}
template <class T, int V, bool kWhole, bool kOnce>
__device__ __forceinline__ void store_group(T* p, int have, const float (&x)[V]) {
  if (kWhole) {
    store_heads<V, kOnce>(p, x);
  } else if (have >= V) {
    T v[V];
    store_heads<V>(v, x);
    __builtin_memcpy(p, v, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < have) store_one(p + i, x[i]);
  }
}
template <int V, bool kWhole, bool kOnce>
__device__ __forceinline__ void store_eight(uint8_t* p, int have, const float (&x)[V]) {
  typedef uint32_t uv __attribute__((ext_vector_type(V / 4)));
  uv v;
#pragma unroll
  for (int i = 0; i < V; i += 4) v[i / 4] = pack_e4m3(x[i], x[i + 1], x[i + 2], x[i + 3]);
  if (kWhole) {
    store_vec<kOnce, uv>(p, v);
  } else if (have >= V) {
    __builtin_memcpy(p, &v, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < have) p[i] = (uint8_t)(v[i / 4] >> (8 * (i % 4)));
  }
}

// kLanes threads a row, kGroups groups of V values a thread.  A block is 256
// threads (a row, or several in a wave or part of one each), or a row's 512 or 1024.
template <class T, int kGroups, int kLanes, bool kWhole, bool kOnce>
__global__ __launch_bounds__(kLanes < 256 ? 256 : kLanes) void k_norm(const NormArgs p) {
  constexpr int V = 16 / sizeof(T);
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  constexpr int kWaves = kLanes < 64 ? 1 : kLanes / 64;
  __shared__ uint32_t shared[2 * kWaves];
  const int i = threadIdx.x % kLanes, wave = i / 64;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
  if (kRows > 1 && row >= p.n_rows) return;   // (a block of one row is never past the end)
  const T* x = (const T*)p.x + row * p.x_row;
  // A row's last group, if it is not whole, begins V before the row's end, so that it is one access too (50000 x 1283 bfloat16
  // with its sum 101 us, 162 by elements).  Its first values are the group before's as well: both store the same, one counts them.
  const auto first = [&](int u) { return (u * kLanes + i) * V; };
  const auto in_row = [&](int u) { return first(u) < p.width; };
  const int last = p.width > V ? p.width - V : 0, have = p.width < V ? p.width : V;
  const auto place = [&](int u) { return kWhole || first(u) < last ? first(u) : last; };
  float h[kGroups][V];
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int at = place(u);
#pragma unroll
    for (int j = 0; j < V; ++j) h[u][j] = 0.f;
    if (in_row(u)) load_group<T, V, kWhole, kOnce>(x + at, have, h[u]);
  }
  if (p.residual) {
    const T* r = (const T*)p.residual + row * p.residual_row;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int at = place(u);
      if (in_row(u)) {
        float a[V];
        load_group<T, V, kWhole, kOnce>(r + at, have, a);
#pragma unroll
        for (int j = 0; j < V; ++j) h[u][j] += a[j];
      }
    }
  }
  if (p.total) {
    if constexpr (!kWhole && kWaves > 1) __syncthreads();   // (it may be an input; waves share a row's last bytes)
    T* t = (T*)p.total + row * p.total_row;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int at = place(u);
      if (in_row(u)) store_group<T, V, kWhole, kOnce>(t + at, have, h[u]);
    }
  }
  if (p.norm) {
    float q = 0.f;
#pragma unroll
    for (int u = 0; u < kGroups; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float a = kWhole || j >= first(u) - place(u) ? h[u][j] : 0.f;
        q = __builtin_fmaf(a, a, q);
      }
    q = sum_lanes<kLanes>(q);
    if constexpr (kWaves > 1) {
      if (i % 64 == 0) shared[wave] = __float_as_uint(q);
      __syncthreads();
      q = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) q += __uint_as_float(shared[w]);
    }
    const float r = reciprocal_root_of(__builtin_fmaf(q, p.inv_width, p.eps));
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int at = place(u);
      if (in_row(u)) {
        float g[V];
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = 1.f;
        if (p.gain) {
          if (kWhole || have == V) {
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = p.gain[at + j];
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j) g[j] = j < have ? p.gain[j] : 0.f;
          }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) h[u][j] = h[u][j] * r * g[j];
      }
    }
  }
  if (!p.eight) {
    T* o = (T*)p.out + row * p.out_row;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int at = place(u);
      if (in_row(u)) store_group<T, V, kWhole, kOnce>(o + at, have, h[u]);
    }
    return;
  }
  // magnitudes as integers: one that is not finite is the largest
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < kGroups; ++u)
#pragma unroll
    for (int j = 0; j < V; ++j) top = max(top, __float_as_uint(h[u][j]) & 0x7fffffffu);
  top = max_lanes<kLanes>(top);
  if constexpr (kWaves > 1) {
    if (i % 64 == 0) shared[kWaves + wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = max(top, shared[kWaves + w]);
  }
  const float scale = top < 0x7f800000u ? fmaxf(__uint_as_float(top) / kE4m3Largest, kE4m3SmallestScale) : __builtin_nanf("");
  const float inv = 1.f / scale;
  if (i == 0) p.out_scale[row] = scale;
  uint8_t* o = (uint8_t*)p.out + row * p.out_row;
#pragma unroll
  for (int u = 0; u < kGroups; ++u) {
    const int at = place(u);
    if (in_row(u)) {
#pragma unroll
      for (int j = 0; j < V; ++j) {   // the quotient, correctly rounded: the product and one step with its remainder
        const float q = h[u][j] * inv;
        h[u][j] = __builtin_fmaf(__builtin_fmaf(-q, scale, h[u][j]), inv, q);
      }
      store_eight<V, kWhole, kOnce>(o + at, have, h[u]);
    }
  }
}

constexpr int64_t kMostBlocks = 1 << 21;   // (of 1024 threads: below 2^32 in all)

template <class T, int kGroups, int kLanes, bool kWhole, bool kOnce>
void launch(NormArgs p, hipStream_t stream) {
  constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;
  constexpr int64_t kRowsMost = kMostBlocks * kRows;
  const int64_t n = p.n_rows;
  const int64_t es = sizeof(T);
  for (int64_t r = 0; r < n; r += kRowsMost) {
    p.n_rows = n - r < kRowsMost ? n - r : kRowsMost;
    k_norm<T, kGroups, kLanes, kWhole, kOnce><<<(unsigned)((p.n_rows + kRows - 1) / kRows), kLanes < 256 ? 256 : kLanes, 0, stream>>>(p);
    p.x = (const char*)p.x + kRowsMost * p.x_row * es;
    if (p.residual) p.residual = (const char*)p.residual + kRowsMost * p.residual_row * es;
    if (p.total) p.total = (char*)p.total + kRowsMost * p.total_row * es;
    p.out = (char*)p.out + kRowsMost * p.out_row * (p.eight ? 1 : es);
    if (p.out_scale) p.out_scale += kRowsMost;
  }
}

// Bytes read and written from which they go past the caches (a copy of them does not stay there anyway): 16384 x 4096 float32
// to 8 bits, 336 MB, 56 us against 60; 10403 x 4096 bfloat16, 128 MB, 23 against 22.
constexpr int64_t kOnceBytes = 192 << 20;

// Narrow rows in parts of a wave (70920 x 16 bfloat16 9 us, 18 in waves), a
// row in one wave up to two groups a lane, rows that are not of whole groups
// up to eight (5741 x 1283 float32 21 us); else in a block
// (196608 x 2048 bfloat16 with its sum 468 us, 497 in waves; 16384 x 4096
// float32 to 8 bits 53 us in blocks of 512, 56 of 256 and 66 of 1024).
template <class T, bool kWhole, bool kOnce>
void launch_groups(const NormArgs& p, hipStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const int groups = (p.width + V - 1) / V;
  if (groups <= 8) return launch<T, 1, 8, kWhole, kOnce>(p, stream);
  if (groups <= 32) return launch<T, 1, 32, kWhole, kOnce>(p, stream);
  if (groups <= 64) return launch<T, 1, 64, kWhole, kOnce>(p, stream);
  if (groups <= 128) return launch<T, 2, 64, kWhole, kOnce>(p, stream);
  if constexpr (!kWhole) {
    if (groups <= 256) return launch<T, 4, 64, kWhole, kOnce>(p, stream);
    if (groups <= 512) return launch<T, 8, 64, kWhole, kOnce>(p, stream);
  } else {
    if (groups <= 256) return launch<T, 1, 256, kWhole, kOnce>(p, stream);
    if (groups <= 512) return launch<T, 2, 256, kWhole, kOnce>(p, stream);
  }
  if (groups <= 1024) return launch<T, 2, 512, kWhole, kOnce>(p, stream);
  if (groups <= 2048) return launch<T, 4, 512, kWhole, kOnce>(p, stream);
  if (groups <= 4096) return launch<T, 4, 1024, kWhole, kOnce>(p, stream);
  launch<T, 8, 1024, kWhole, kOnce>(p, stream);
}

template <class T>
void launch_norm(const NormArgs& p, bool whole, hipStream_t stream) {
  const int64_t bytes = (int64_t)sizeof(T) * (1 + (p.residual != nullptr) + (p.total != nullptr)) + (p.eight ? 1 : sizeof(T));
  if (whole && p.n_rows * p.width >= kOnceBytes / bytes) launch_groups<T, true, true>(p, stream);
  else if (whole) launch_groups<T, true, false>(p, stream);
  else launch_groups<T, false, false>(p, stream);
}

int check_width(int64_t n_rows, int width, int dtype, const char* who) {
  if (dtype != GC_F32 && dtype != GC_BF16) return fail(GC_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
  if (n_rows < 0 || n_rows > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: n_rows=%lld outside [0, 2^31-1]", who, (long long)n_rows);
  if (width < 1 || width > GC_MAX_WIDTH) return fail(GC_ERR_CAPACITY, "%s: width=%d outside [1, %d]", who, width, GC_MAX_WIDTH);
  return GC_OK;
}

constexpr int64_t kMostStride = (int64_t)1 << 40;

// out and out_scale of either call against each other.
int check_eight(const gc_rows* out, const float* out_scale, int64_t n_rows, int width, const char* who) {
  if (!out_scale) return fail(GC_ERR_ARG, "%s: out_scale is null", who);
  if (reinterpret_cast<uintptr_t>(out_scale) & 3) return fail(GC_ERR_ALIGN, "%s: out_scale misaligned", who);
  if (rows_overlap(*out, n_rows, width, 1, out_scale, (size_t)n_rows * 4)) return fail(GC_ERR_ALIAS, "%s: out overlaps out_scale", who);
  return GC_OK;
}

// Launches what the arguments ask for: groups of 16 bytes where every tensor allows it.
void run_norm(const NormArgs& p, int dtype, hipStream_t stream) {
  const int es = dtype_bytes(dtype), V = 16 / es;
  const auto fits = [&](const void* data, int64_t stride, int bytes, int e) { return !data || rows_aligned({(void*)data, stride}, p.n_rows, bytes, e); };
  const bool whole = p.width % V == 0 && fits(p.x, p.x_row, 16, es) && fits(p.residual, p.residual_row, 16, es) &&
                    fits(p.total, p.total_row, 16, es) && fits(p.out, p.out_row, p.eight ? V : 16, p.eight ? 1 : es);
  if (dtype == GC_F32) launch_norm<float>(p, whole, stream);
  else launch_norm<uint16_t>(p, whole, stream);
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" int gc_add_rms_norm(const gc_rows* x, const gc_rows* residual, int64_t n_rows, int width, int dtype,
                               const float* gain, double eps, const gc_rows* total, const gc_rows* out, int out_dtype,
                               float* out_scale, hipStream_t stream) {
  clear_error();
  const char* who = "gc_add_rms_norm";
  int rc = check_width(n_rows, width, dtype, who);
  if (rc) return rc;
  if (out_dtype != dtype && out_dtype != GC_E4M3) return fail(GC_ERR_DTYPE, "%s: out_dtype %d with dtype %d", who, out_dtype, dtype);
  // (an eps that is 0 in float32 would make NaN of rows of zeros, one that is infinite 0 of all)
  if (!(eps >= 0) || !std::isfinite((float)eps) || (eps > 0 && (float)eps == 0.f))
    return fail(GC_ERR_ARG, "%s: eps=%g must be finite and not negative in float32, and above 0 there unless it is 0", who, eps);
  if (out_dtype != GC_E4M3 && out_scale) return fail(GC_ERR_ARG, "%s: out_scale is given without 8-bit rows", who);
  if (n_rows == 0) return GC_OK;
  if ((rc = check_rows(x, dtype, false, kMostStride, "x", who)) ||
      (residual && (rc = check_rows(residual, dtype, false, kMostStride, "residual", who))) ||
      (total && ((rc = check_rows(total, dtype, false, kMostStride, "total", who)) ||
                 (rc = check_rows_out(*total, n_rows, width, "total", who)))) ||
      (rc = check_rows(out, out_dtype, false, kMostStride, "out", who)) || (rc = check_rows_out(*out, n_rows, width, "out", who)))
    return rc;
  const bool eight = out_dtype == GC_E4M3;
  if (eight && (rc = check_eight(out, out_scale, n_rows, width, who))) return rc;
  if (reinterpret_cast<uintptr_t>(gain) & 3) return fail(GC_ERR_ALIGN, "%s: gain misaligned", who);
  const int64_t es = dtype_bytes(dtype), eo = eight ? 1 : es;
  const size_t scale_bytes = eight ? (size_t)n_rows * 4 : 0, gain_bytes = gain ? (size_t)width * 4 : 0;
  const gc_rows* in[2] = {x, residual};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    const char* name = i ? "residual" : "x";
    if (rows_overlap(*out, n_rows, width, eo, *in[i], n_rows, width, es) && (eight || !same_rows(*out, n_rows, *in[i], n_rows)))
      return fail(GC_ERR_ALIAS, "%s: out overlaps %s", who, name);
    if (total && rows_overlap(*total, n_rows, width, es, *in[i], n_rows, width, es) && !same_rows(*total, n_rows, *in[i], n_rows))
      return fail(GC_ERR_ALIAS, "%s: total overlaps %s", who, name);
    if (rows_overlap(*in[i], n_rows, width, es, out_scale, scale_bytes)) return fail(GC_ERR_ALIAS, "%s: out_scale overlaps %s", who, name);
  }
  if (total && (rows_overlap(*total, n_rows, width, es, *out, n_rows, width, eo) ||
                rows_overlap(*total, n_rows, width, es, out_scale, scale_bytes)))
    return fail(GC_ERR_ALIAS, "%s: total overlaps out or out_scale", who);
  if (rows_overlap(*out, n_rows, width, eo, gain, gain_bytes) || (total && rows_overlap(*total, n_rows, width, es, gain, gain_bytes)) ||
      overlaps(out_scale, scale_bytes, gain, gain_bytes))
    return fail(GC_ERR_ALIAS, "%s: an output overlaps gain", who);
  NormArgs p = {};
  p.x = x->data, p.x_row = x->stride;
  if (residual) p.residual = residual->data, p.residual_row = residual->stride;
  if (total) p.total = total->data, p.total_row = total->stride;
  p.out = out->data, p.out_row = out->stride, p.out_scale = out_scale;
  p.gain = gain;
  p.n_rows = n_rows, p.width = width;
  p.norm = 1, p.eight = eight;
  p.eps = (float)eps, p.inv_width = 1.f / (float)width;
  run_norm(p, dtype, stream);
  return after_launch(stream, who);
}

extern "C" int gc_quantize_rows(const gc_rows* x, int64_t n_rows, int width, int dtype, const gc_rows* out,
                                float* out_scale, hipStream_t stream) {
  clear_error();
  const char* who = "gc_quantize_rows";
  int rc = check_width(n_rows, width, dtype, who);
  if (rc || n_rows == 0) return rc;
  if ((rc = check_rows(x, dtype, false, kMostStride, "x", who)) || (rc = check_rows(out, GC_E4M3, false, kMostStride, "out", who)) ||
      (rc = check_rows_out(*out, n_rows, width, "out", who)) || (rc = check_eight(out, out_scale, n_rows, width, who)))
    return rc;
  const int64_t es = dtype_bytes(dtype);
  if (rows_overlap(*out, n_rows, width, 1, *x, n_rows, width, es) || rows_overlap(*x, n_rows, width, es, out_scale, (size_t)n_rows * 4))
    return fail(GC_ERR_ALIAS, "%s: out or out_scale overlaps x", who);
  NormArgs p = {};
  p.x = x->data, p.x_row = x->stride;
  p.out = out->data, p.out_row = out->stride, p.out_scale = out_scale;
  p.n_rows = n_rows, p.width = width;
  p.eight = 1;
  run_norm(p, dtype, stream);
  return after_launch(stream, who);
}
