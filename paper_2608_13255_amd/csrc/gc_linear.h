// Matrix products with what follows them: arguments, operand types and the
// epilogue that all variants share.
#pragma once

#include "gc_rows.h"

namespace gc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
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
  int out_whole, residual_whole; // 16 bytes of a row may be accessed at once
  int parts;                     // of the inner dimension
  int part_bytes;                // of a row in a part (the last one may be shorter)
  float* partial;                // [parts][n_rows][n_out, or 2 n_out]
};

// Activations, in float32.
__device__ __forceinline__ float activation(float p, int act) {
  if (act == GC_ACT_SILU) return p / (1.f + expf(-p));
  if (act == GC_ACT_GELU) return 0.5f * p * (1.f + erff(p * 0.70710678118654752f));
  // (1 + tanh u) / 2 = 1 / (1 + e^(-2u))
  if (act == GC_ACT_GELU_TANH) return p / (1.f + expf(-1.5957691216057308f * (p + 0.044715f * p * p * p)));
  return p;
}

// kCount consecutive outputs of one row, from column n (the last ones may lie past the end): the sums' epilogue.
// gate: with gated products those of the value rows; otherwise unused.
template <int kCount>
__device__ __forceinline__ void load_floats(const float* p, int have, float fill, float (&v)[kCount]) {
#pragma unroll
  for (int i = 0; i < kCount; ++i) v[i] = p && i < have ? p[i] : fill;
}
template <int kCount>
__device__ __forceinline__ void finish(const LinearArgs& p, int64_t m, int n, float (&a)[kCount], float (&b)[kCount]) {
  const int have = p.n_out - n;
  if (m >= p.n_rows || have <= 0) return;
  const float xs = p.x_scale ? p.x_scale[m] : 1.f;
  float s[kCount];
  if (p.x_scale || p.w_scale) {
    load_floats<kCount>(p.w_scale ? p.w_scale + n : nullptr, have, 1.f, s);
#pragma unroll
    for (int i = 0; i < kCount; ++i) a[i] = a[i] * xs * s[i];
  }
  if (p.bias) {
    load_floats<kCount>(p.bias + n, have, 0.f, s);
#pragma unroll
    for (int i = 0; i < kCount; ++i) a[i] += s[i];
  }
#pragma unroll
  for (int i = 0; i < kCount; ++i) a[i] = activation(a[i], p.act);
  if (p.gated) {
    if (p.x_scale || p.w_scale) {
      load_floats<kCount>(p.w_scale ? p.w_scale + p.n_out + n : nullptr, have, 1.f, s);
#pragma unroll
      for (int i = 0; i < kCount; ++i) b[i] = b[i] * xs * s[i];
    }
    if (p.bias) {
      load_floats<kCount>(p.bias + p.n_out + n, have, 0.f, s);
#pragma unroll
      for (int i = 0; i < kCount; ++i) b[i] += s[i];
    }
#pragma unroll
    for (int i = 0; i < kCount; ++i) a[i] *= b[i];
  }
  const int es = p.out_f32 ? 4 : 2;
  if (p.residual) {
    const char* r = p.residual + m * p.residual_row + (int64_t)n * es;
    if (p.out_f32) {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (i < have) a[i] += ((const float*)r)[i];
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i)
        if (i < have) a[i] += load_one((const uint16_t*)r + i);
    }
  }
  char* o = p.out + m * p.out_row + (int64_t)n * es;
  if (p.out_f32) {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (i < have) ((float*)o)[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      if (i < have) store_one((uint16_t*)o + i, a[i]);
  }
}

// Operand types: what a pair of 16-byte chunks of a row, one in either half
// of the wave's lanes, multiplies.  The order of the products inside is free:
// both operands have the same.
struct F32 {
  static constexpr int kPairs = 1;   // of chunks that a product takes
  typedef f32x4 Frag;
  __device__ __forceinline__ static f32x16 mma(const Frag& w, const Frag& x, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(w[i], x[i], c, 0, 0, 0);
    return c;
  }
};
struct BF16 {
  static constexpr int kPairs = 1;
  typedef bf16x8 Frag;
  __device__ __forceinline__ static f32x16 mma(const Frag& w, const Frag& x, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x, c, 0, 0, 0);
  }
};
struct E4M3 {
  static constexpr int kPairs = 2;
  typedef i32x8 Frag;
  __device__ __forceinline__ static f32x16 mma(const Frag& w, const Frag& x, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, 0, 0, 0);
  }
};

}  // namespace gc
