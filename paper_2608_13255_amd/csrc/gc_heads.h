// Tensors of heads [tokens][heads][dim] with strides: their host checks, and
// loads and stores of a few channels at a time.
#pragma once

#include "gc_common.h"

namespace gc {

// A tensor of heads against its sizes: pointer, alignment and strides.
inline int check_heads(const gc_heads* t, int dtype, const char* name, const char* who) {
  if (!t || !t->data) return fail(GC_ERR_ARG, "%s: %s is null", who, name);
  const int64_t es = dtype_bytes(dtype);
  // a stride of 2^22 elements keeps the byte offsets inside a tile of 64 tokens below 2^31
  if (t->token_stride < 0 || t->head_stride < 0 || t->token_stride > (1 << 22) || t->head_stride > (int64_t)1 << 40)
    return fail(GC_ERR_SHAPE, "%s: %s has strides (%lld, %lld): token strides are 0 to 2^22, head strides not negative", who,
                name, (long long)t->token_stride, (long long)t->head_stride);
  if (!aligned16(t->data) || (t->token_stride * es) % 16 || (t->head_stride * es) % 16)
    return fail(GC_ERR_ALIGN, "%s: %s must be 16-byte aligned with strides of whole 16 bytes", who, name);
  return GC_OK;
}

// The sizes and types that the operators on heads share.
inline int check_head_sizes(int heads, int dim, int dtype, const char* who) {
  if (dtype != GC_F32 && dtype != GC_BF16) return fail(GC_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
  if (heads < 1 || heads > GC_MAX_HEADS) return fail(GC_ERR_CAPACITY, "%s: heads=%d outside [1, %d]", who, heads, GC_MAX_HEADS);
  if (dim < 8 || dim % 8 || dim > GC_MAX_HEAD_DIM)
    return fail(GC_ERR_SHAPE, "%s: dim=%d is not a multiple of 8 in [8, %d]", who, dim, GC_MAX_HEAD_DIM);
  return GC_OK;
}

// Whether two tensors of heads may share bytes.  Their extents decide, except
// that columns of one buffer (equal token strides, each token's span inside
// the stride) are told apart within the stride.
inline bool heads_overlap(const gc_heads& a, int64_t ta, int ha, const gc_heads& b, int64_t tb, int hb, int dim, int dtype) {
  const int64_t es = dtype_bytes(dtype);
  if (ta < 1 || tb < 1) return false;
  const int64_t wa = ((ha - 1) * a.head_stride + dim) * es, wb = ((hb - 1) * b.head_stride + dim) * es;
  const int64_t sa = a.token_stride * es, sb = b.token_stride * es;
  if (!overlaps(a.data, (size_t)((ta - 1) * sa + wa), b.data, (size_t)((tb - 1) * sb + wb))) return false;
  if (sa != sb || sa <= 0 || wa > sa || wb > sa) return true;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.data) - reinterpret_cast<uintptr_t>(a.data));
  const int64_t m = ((d % sa) + sa) % sa;   // b's first column within a's token
  return m < wa || m + wb > sa;
}

inline bool same_heads(const gc_heads& a, const gc_heads& b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

// An output [t][h][dim] of its own: no element is written twice.
inline int check_heads_out(const gc_heads& o, int64_t t, int h, int dim, const char* name, const char* who) {
  const bool token_major = (h == 1 || o.head_stride >= dim) && (t <= 1 || o.token_stride >= (h - 1) * o.head_stride + dim);
  const bool head_major = (t <= 1 || o.token_stride >= dim) && (h == 1 || o.head_stride >= (t - 1) * o.token_stride + dim);
  if (!token_major && !head_major) return fail(GC_ERR_SHAPE, "%s: the strides of %s make its elements overlap", who, name);
  return GC_OK;
}

// ---------------------------------------------------------------------------
// device
// ---------------------------------------------------------------------------

// V channels as floats, one memory access of V * sizeof(T) bytes (at most
// 16); kOnce: data that is not used again soon, past the caches.
template <bool kOnce, class X>
__device__ __forceinline__ X load_vec(const void* p) {
  if constexpr (kOnce) return __builtin_nontemporal_load(reinterpret_cast<const X*>(p));
  else return *reinterpret_cast<const X*>(p);
}
template <bool kOnce, class X>
__device__ __forceinline__ void store_vec(void* p, X x) {
  if constexpr (kOnce) __builtin_nontemporal_store(x, reinterpret_cast<X*>(p));
  else *reinterpret_cast<X*>(p) = x;
}
// V channels as they lie in memory, and as floats.
template <class T, int V>
struct HeadVec;
template <int V>
struct HeadVec<float, V> {
  typedef float type __attribute__((ext_vector_type(V)));
  __device__ __forceinline__ static float at(const type& v, int i) { return v[i]; }
};
template <int V>
struct HeadVec<uint16_t, V> {
  typedef uint32_t type __attribute__((ext_vector_type(V / 2)));
  __device__ __forceinline__ static float at(const type& v, int i) {
    return __uint_as_float((i & 1) ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
  }
};
template <int V, class T>
__device__ __forceinline__ void load_heads(const T* p, float (&x)[V]) {
  const auto v = *reinterpret_cast<const typename HeadVec<T, V>::type*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = HeadVec<T, V>::at(v, i);
}
template <int V, bool kOnce = false>
__device__ __forceinline__ void store_heads(float* p, const float (&x)[V]) {
  typedef float fv __attribute__((ext_vector_type(V)));
  fv v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = x[i];
  store_vec<kOnce, fv>(p, v);
}
// Two floats to a pair of bfloat16, round to nearest even (a NaN stays one).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v;
  v.x = (__bf16)lo;
  v.y = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}
template <int V, bool kOnce = false>
__device__ __forceinline__ void store_heads(uint16_t* p, const float (&x)[V]) {
  typedef uint32_t uv __attribute__((ext_vector_type(V / 2)));
  uv v;
#pragma unroll
  for (int i = 0; i < V; i += 2) v[i / 2] = pack_bf16(x[i], x[i + 1]);
  store_vec<kOnce, uv>(p, v);
}

}  // namespace gc
