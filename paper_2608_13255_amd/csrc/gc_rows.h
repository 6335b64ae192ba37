// Rows [rows][columns] with a stride: their host checks, and 8-bit values.
#pragma once

#include "gc_heads.h"

namespace gc {

inline int row_type_bytes(int dtype) { return dtype == GC_E4M3 ? 1 : dtype_bytes(dtype); }

// Rows against their sizes: pointer, its alignment (of an element, or of 16 bytes with whole 16 bytes a row) and stride.
inline int check_rows(const gc_rows* t, int dtype, bool whole16, int64_t most_stride, const char* name, const char* who) {
  if (!t || !t->data) return fail(GC_ERR_ARG, "%s: %s is null", who, name);
  if (t->stride < 0 || t->stride > most_stride)
    return fail(GC_ERR_SHAPE, "%s: %s has stride %lld outside [0, %lld]", who, name, (long long)t->stride, (long long)most_stride);
  const int64_t es = row_type_bytes(dtype);
  if (whole16 && (!aligned16(t->data) || (t->stride * es) % 16))
    return fail(GC_ERR_ALIGN, "%s: %s must be 16-byte aligned with a stride of whole 16 bytes", who, name);
  if (reinterpret_cast<uintptr_t>(t->data) % es) return fail(GC_ERR_ALIGN, "%s: %s is not aligned to its elements", who, name);
  return GC_OK;
}

// An output's rows share no memory.
inline int check_rows_out(const gc_rows& o, int64_t rows, int64_t width, const char* name, const char* who) {
  if (rows > 1 && o.stride < width) return fail(GC_ERR_SHAPE, "%s: the stride of %s makes its rows overlap", who, name);
  return GC_OK;
}

// Whether the rows may be accessed 16 bytes at a time (rows of `es`-byte elements whose groups of `group` fill that).
inline bool rows_aligned(const gc_rows& t, int64_t rows, int64_t bytes, int es) {
  return reinterpret_cast<uintptr_t>(t.data) % bytes == 0 && (rows <= 1 || (t.stride * es) % bytes == 0);
}

// Whether two matrices of rows may share bytes.  Their extents decide, except
// that columns of one buffer (equal strides in bytes, each row inside the
// stride) are told apart within the stride.
inline bool rows_overlap(const gc_rows& a, int64_t na, int64_t wa, int64_t ea, const gc_rows& b, int64_t nb, int64_t wb, int64_t eb) {
  if (na < 1 || nb < 1) return false;
  wa *= ea, wb *= eb;
  const int64_t sa = a.stride * ea, sb = b.stride * eb;
  if (!overlaps(a.data, (size_t)((na - 1) * sa + wa), b.data, (size_t)((nb - 1) * sb + wb))) return false;
  if (sa != sb || sa <= 0 || wa > sa || wb > sa) return true;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.data) - reinterpret_cast<uintptr_t>(a.data));
  const int64_t m = ((d % sa) + sa) % sa;   // b's first column within a's row
  return m < wa || m + wb > sa;
}

inline bool rows_overlap(const gc_rows& a, int64_t na, int64_t wa, int64_t ea, const void* p, size_t bytes) {
  return na > 0 && overlaps(a.data, (size_t)((na - 1) * a.stride * ea + wa * ea), p, bytes);
}

inline bool same_rows(const gc_rows& a, int64_t na, const gc_rows& b, int64_t nb) {
  return a.data == b.data && na == nb && (na <= 1 || a.stride == b.stride);
}

// ---------------------------------------------------------------------------
// device
// ---------------------------------------------------------------------------

constexpr float kE4m3Largest = 448.f;
constexpr float kE4m3SmallestScale = 0x1p-126f;

// Four floats, none above 464 in magnitude, to 8 bits each (the hardware's rounding to nearest even; a NaN stays one).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// One value as it lies in memory, to a float and back.
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_one(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_one(uint16_t* p, float x) { *p = (uint16_t)pack_bf16(x, x); }

}  // namespace gc
