// Matrix products with what follows them: arguments, operand types and the
// epilogue that all variants share.
#pragma once

#include "gc_rows.h"

namespace gc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const char *x, *w;
  int64_t x_row, w_row;          // bytes
  const float *x_scale, *w_scale, *bias;
  const char* residual;
  char* out;
  int64_t residual_row, out_row; // bytes
  int64_t n_rows;
  int n_out, row_bytes;          // row_bytes: of n_in operands
  int act, gated, out_f32;
  int whole;                     // groups of 8 outputs may be accessed as 16 bytes
  int parts;                     // of the inner dimension
  int part_bytes;                // of a row in a part, a multiple of kStepBytes (the last one may be shorter)
  float* partial;                // sums of the parts: [parts][n_rows][partial_cols, or 2 partial_cols]
  int64_t partial_part;          // floats of one part
  int partial_cols;              // n_out, and up to a multiple of 8
};

constexpr int kStepBytes = 128;   // of a row that a tile reads at a time

// p * 1 / (1 + e^-u): u = p, or 2 sqrt(2 / pi) (p + 0.044715 p^3), since (1 + tanh v) / 2 = 1 / (1 + e^(-2 v)).
__device__ __forceinline__ float times_logistic(float p, float u_log2e) {
  return p * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-u_log2e));
}
// p times the normal distribution function of p.  The tail beyond |p| is e^(-p^2 / 2) t P(t) / 2 with
// t = 1 / (1 + 0.38 |p| / sqrt 2) and P fitted to e^(z^2) erfc(z) / t by least squares at Chebyshev nodes of t, weighted
// towards the largest relative error (3.1e-8 up to |p| = 14.5, from where on the tail is no float32).
__device__ __forceinline__ float gelu(float p) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(p), 0.26870057685088805f, 1.f));
  float q = 0.059048961848020554f;
  q = __builtin_fmaf(q, t, -0.2626957595348358f);
  q = __builtin_fmaf(q, t, 0.36475491523742676f);
  q = __builtin_fmaf(q, t, -0.16252949833869934f);
  q = __builtin_fmaf(q, t, 0.23080290853977203f);
  q = __builtin_fmaf(q, t, 0.13829964399337769f);
  q = __builtin_fmaf(q, t, 0.20400194823741913f);
  q = __builtin_fmaf(q, t, 0.21390503644943237f);
  q = __builtin_fmaf(q, t, 0.2144118696451187f);
  const float tail = 0.5f * __builtin_amdgcn_exp2f(p * p * -0.72134752044448170f) * (t * q);
  return p * (p > 0.f ? 1.f - tail : tail);
}
template <int kCount>
__device__ __forceinline__ void activate(float (&p)[kCount], int act) {
  if (act == GC_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) p[i] = times_logistic(p[i], p[i] * 1.4426950408889634f);
  } else if (act == GC_ACT_GELU_TANH) {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      p[i] = times_logistic(p[i], p[i] * __builtin_fmaf(p[i] * p[i], 0.10294323970f, 2.3022081985f));
  } else if (act == GC_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) p[i] = gelu(p[i]);
  }
}

// Eight consecutive columns of the output, all inside it: what the epilogue has of them.
struct Columns {
  int n;
  float scale[8], bias[8], value_scale[8], value_bias[8];
  __device__ __forceinline__ static void load(const float* p, float fill, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fill;
    if (!p) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
  }
  template <bool kGated>
  __device__ __forceinline__ void init(const LinearArgs& p, int first) {
    n = first;
    load(p.w_scale ? p.w_scale + n : nullptr, 1.f, scale);
    load(p.bias ? p.bias + n : nullptr, 0.f, bias);
    if (kGated) {
      load(p.w_scale ? p.w_scale + p.n_out + n : nullptr, 1.f, value_scale);
      load(p.bias ? p.bias + p.n_out + n : nullptr, 0.f, value_bias);
    }
  }
};

// What the epilogue reads of a row: asked for before it is needed, and before the rows in front of it are stored, since the
// output may be the residual.
struct RowAhead {
  u32x4 add[2];
  float scale;
  __device__ __forceinline__ void load(const LinearArgs& p, int64_t m, int n) {
    if (p.residual) {
      const char* r = p.residual + m * p.residual_row + (int64_t)n * (p.out_f32 ? 4 : 2);
      add[0] = *reinterpret_cast<const u32x4*>(r);
      if (p.out_f32) add[1] = *reinterpret_cast<const u32x4*>(r + 16);
    }
    if (p.x_scale) scale = p.x_scale[m];
  }
};

// The sums a (and b of the value rows) of eight columns of row m to the output, 16 bytes at a time.  kOnce: past the caches.
template <bool kGated, bool kOnce = false>
__device__ __forceinline__ void finish(const LinearArgs& p, const Columns& c, int64_t m, const RowAhead& row, float (&a)[8], float (&b)[8]) {
  if (p.x_scale || p.w_scale) {
    const float xs = p.x_scale ? row.scale : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = a[i] * xs * c.scale[i];
    if (kGated) {
#pragma unroll
      for (int i = 0; i < 8; ++i) b[i] = b[i] * xs * c.value_scale[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] += c.bias[i];
  activate<8>(a, p.act);
  if (kGated) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] *= b[i] + c.value_bias[i];
  }
  char* o = p.out + m * p.out_row + (int64_t)c.n * (p.out_f32 ? 4 : 2);
  if (p.out_f32) {
    if (p.residual) {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] += __uint_as_float(row.add[i / 4][i % 4]);
    }
    store_heads<8, kOnce>((float*)o, a);
  } else {
    if (p.residual) {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] += HeadVec<uint16_t, 8>::at(row.add[0], i);
    }
    store_heads<8, kOnce>((uint16_t*)o, a);
  }
}

// The same for one column.
struct Column {
  int n;
  float scale, bias, value_scale, value_bias;
  template <bool kGated>
  __device__ __forceinline__ void init(const LinearArgs& p, int at) {
    n = at;
    scale = p.w_scale ? p.w_scale[n] : 1.f;
    bias = p.bias ? p.bias[n] : 0.f;
    if (kGated) {
      value_scale = p.w_scale ? p.w_scale[p.n_out + n] : 1.f;
      value_bias = p.bias ? p.bias[p.n_out + n] : 0.f;
    }
  }
};
struct OneAhead {
  float add, scale;
  __device__ __forceinline__ void load(const LinearArgs& p, int64_t m, int n) {
    add = 0.f, scale = 1.f;
    if (p.residual) {
      const char* r = p.residual + m * p.residual_row;
      add = p.out_f32 ? ((const float*)r)[n] : load_one((const uint16_t*)r + n);
    }
    if (p.x_scale) scale = p.x_scale[m];
  }
};
template <bool kGated>
__device__ __forceinline__ void finish_one(const LinearArgs& p, const Column& c, int64_t m, const OneAhead& row, float sum, float value) {
  float a[1] = {sum}, b = value;
  if (p.x_scale || p.w_scale) {
    a[0] = a[0] * row.scale * c.scale;
    if (kGated) b = b * row.scale * c.value_scale;
  }
  a[0] += c.bias;
  activate<1>(a, p.act);
  if (kGated) a[0] *= b + c.value_bias;
  if (p.residual) a[0] += row.add;
  if (p.out_f32) ((float*)(p.out + m * p.out_row))[c.n] = a[0];
  else store_one((uint16_t*)(p.out + m * p.out_row) + c.n, a[0]);
}

// Operand types.  A product takes kBlock rows of either operand; a fragment of
// them is kChunks 16-byte chunks a lane, of row lane % kBlock and with the lanes'
// groups side by side.  Which of a row's products a fragment holds where is
// free: both operands have them alike.  Of an accumulator's four consecutive elements q the lane holds
// weight rows kStride q + 4 (lane / kBlock) .. + 3 for row lane % kBlock of x.
struct Blocks32 {
  static constexpr int kBlock = 32, kQuads = 4, kStride = 8;
  typedef f32x16 Acc;
};
struct Blocks16 {
  static constexpr int kBlock = 16, kQuads = 1, kStride = 16;
  typedef f32x4 Acc;
};
struct F32 : Blocks16 {
  static constexpr int kChunks = 1, kProducts = 4;   // products of a pair of fragments
  static constexpr bool kTotals = true;
  typedef f32x4 Frag;
  __device__ __forceinline__ static Acc mma(const Frag& w, const Frag& x, Acc c, int i) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[i], c, 0, 0, 0);
  }
};
struct BF16 : Blocks16 {
  static constexpr int kChunks = 1, kProducts = 1;
  static constexpr bool kTotals = false;
  typedef bf16x8 Frag;
  __device__ __forceinline__ static Acc mma(const Frag& w, const Frag& x, Acc c, int) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0);
  }
};
// The 8-bit products add their terms to fewer bits than float32 has: over rows of 64 to 4096 they are 1.2e-5 of the products' root
// sum of squares off in the 2-norm, 7e-5 with channels of 100 times the others' size, whatever the sum itself is.  A bfloat16
// result is rounded by 1.7e-3 of itself, so it takes them; for a float32 result the operands become bfloat16 first, which
// holds them exactly.
struct E4M3Exact : Blocks32 {
  static constexpr int kChunks = 1, kProducts = 2;
  static constexpr bool kTotals = false;
  typedef u32x4 Frag;
  __device__ __forceinline__ static bf16x8 half(const Frag& f, int i) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    bf16x8 r;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + j], 1.f, false);
      const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * i + j], 1.f, true);
      r[4 * j] = lo[0], r[4 * j + 1] = lo[1], r[4 * j + 2] = hi[0], r[4 * j + 3] = hi[1];
    }
    return r;
  }
  __device__ __forceinline__ static Acc mma(const Frag& w, const Frag& x, Acc c, int i) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(half(w, i), half(x, i), c, 0, 0, 0);
  }
};
struct E4M3 : Blocks32 {
  static constexpr int kChunks = 2, kProducts = 1;
  static constexpr bool kTotals = false;
  typedef i32x8 Frag;
  __device__ __forceinline__ static Acc mma(const Frag& w, const Frag& x, Acc c, int) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0);   // (no scales: ones)
  }
};

}  // namespace gc
