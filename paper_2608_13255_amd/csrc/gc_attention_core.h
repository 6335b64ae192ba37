// Attention on the matrix units: what one wave does with one tile of keys.
//
// A wave holds 32 query rows (columns of the products) and works on S^T = K Q^T
// and O^T = V^T P^T.  In both products the accumulator's column is the query
// row, lane % 32, so the row's maximum, sum and rescaling factor are one
// register each and the weights P^T are used as the second product's operand
// in the lane that computed them.  An accumulator's element i of half h
// (h = lane / 32) is row 8 (i / 4) + 4 h + i % 4; the order of the keys inside
// a product is free, so the values are read in the order in which the weights lie.
//
// K and V tiles lie in LDS as rows of 16-byte chunks, chunk c of row r at
// place c ^ f(r): with f below, 16 rows' same chunk lie in 16 different
// places of the 256 bytes that the banks span, and so do four rows' same
// four chunks.
#pragma once

#include "gc_attention_plan.h"

namespace gc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttentionArgs {
  const void *q, *k, *v;
  void* out;
  float* lse;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  const AttentionItem* items;
  int heads, kv_heads, group, dim;
  int total_q, total_k;
  int causal;
  float scale;
  float* partial;       // per slot and kv head: [tile_rows][dim padded] weighted sums, then [tile_rows][2] maxima and sums
  uint32_t* counters;   // per group and kv head: parts that are done
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Byte of chunk c of row r in a tile of kChunks chunks a row.  Only the low
// bits of the chunk are permuted, by their exclusive or with f(r).
template <int kChunks>
__device__ __forceinline__ int place(int row, int chunk) {
  constexpr int kLow = kChunks % 16 == 0 ? 16 : kChunks % 8 == 0 ? 8 : 4;
  const int f = kLow == 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : kLow == 8 ? ((row & 2) << 1) | ((row >> 2) & 3) : (row >> 2) & 3;
  return row * (kChunks * 16) + (chunk & ~(kLow - 1)) * 16 + ((chunk & (kLow - 1)) ^ f) * 16;
}

typedef __attribute__((address_space(3))) void LdsVoid;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The larger of a lane's value and that of the lane 32 away; their sum.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Copies kKeys rows of a K or V tensor to LDS with the swizzle, straight from
// memory (buffer loads to LDS: 16 bytes a lane, places in lane order).
// Rows past the sequence's last key, and channels past dim, arrive as
// zeros: the buffer's range ends there.
template <class T, int kDim, int kKeys, int kWaves>
struct TileLoader {
  static constexpr int kChunks = kDim * (int)sizeof(T) / 16;
  static constexpr int kLoads = kKeys * kChunks / 64;     // of a wave's 64 lanes
  static constexpr int kMine = (kLoads + kWaves - 1) / kWaves;
  static_assert(kKeys * kChunks % 64 == 0, "whole loads");
  const char* base;       // the head's first key
  int64_t stride;         // bytes
  int row_bytes;
  uint32_t offset[kMine];

  __device__ __forceinline__ void init(const void* p, int64_t first_token, int64_t token_stride, int64_t head_off, int dim,
                                       int wave, int lane) {
    stride = token_stride * (int64_t)sizeof(T);
    base = (const char*)p + first_token * stride + head_off * (int64_t)sizeof(T);
    row_bytes = dim * (int)sizeof(T);
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const int at = (wave + n * kWaves) * 64 + lane;
      // the chunk that lies at this place: the exclusive or is its own inverse
      const int row = at / kChunks, chunk = place<kChunks>(row, at % kChunks) / 16 - row * kChunks;
      offset[n] = chunk * 16 < row_bytes ? (uint32_t)row * (uint32_t)stride + (uint32_t)chunk * 16u : 0x7ffffff0u;
    }
  }

  // keys [first, first + kKeys) of a sequence of k_len, first < k_len
  __device__ __forceinline__ void load(char* lds, int first, int k_len, int wave) const {
    const int rows = k_len - first < kKeys ? k_len - first : kKeys;
    const int bytes = (rows - 1) * (int)stride + row_bytes;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + first * stride), 0, bytes, 0x00027000);
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const int i = wave + n * kWaves;
      if (kLoads % kWaves == 0 || i < kLoads)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid*)(lds + i * 1024), 16, offset[n], 0, 0, 0);
    }
  }
};

// The query rows of a wave: row n * 32 + lane % 32 of its tile for n < kBlocks.
struct RowOf {
  int64_t token;
  int head;
  int limit;     // keys [0, limit) are seen
  bool live;
};
__device__ __forceinline__ RowOf row_of(const AttentionArgs& p, const AttentionItem& it, int kv_head, int row) {
  RowOf r;
  r.live = row < it.rows;
  const int c = r.live ? row : it.rows - 1;
  const int tok = c / p.group;
  r.token = (int64_t)it.q_token0 + tok;
  r.head = kv_head * p.group + (c - tok * p.group);
  r.limit = it.k_len;
  if (p.causal) r.limit = tok + it.reach < it.k_len ? tok + it.reach : it.k_len;
  return r;
}

// ---------------------------------------------------------------------------
// bfloat16
// ---------------------------------------------------------------------------
template <class T, int kDim, int kNq, int kKeyBlocks>
struct Core;

template <int kDim, int kNq, int kKeyBlocks>
struct Core<uint16_t, kDim, kNq, kKeyBlocks> {
  static constexpr int kChunks = kDim / 8, kSteps = kDim / 16, kOut = kDim / 32;
  bf16x8 q[kNq][kSteps];
  f32x16 o[kNq][kOut];
  float m[kNq], l[kNq];   // maximum in use (score times scale times log2 e) and this lane's part of the sum

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < kNq; ++n) {
#pragma unroll
      for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][d][i] = 0.f;
      m[n] = -__builtin_inff();
      l[n] = 0.f;
    }
  }

  __device__ __forceinline__ void load_q(int n, const uint16_t* row, int dim, int half) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if ((2 * s + half) * 8 < dim) w = *reinterpret_cast<const u32x4*>(row + (2 * s + half) * 8);
      q[n][s] = __builtin_bit_cast(bf16x8, w);
    }
  }

  // scores of the tile, S^T: key 32 b + 8 (i / 4) + 4 half + i % 4
  __device__ __forceinline__ void scores(const char* kt, int lane, f32x16 (&s)[kNq][kKeyBlocks]) const {
    const int r = lane & 31, half = lane >> 5;
#pragma unroll
    for (int n = 0; n < kNq; ++n)
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][b][i] = 0.f;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b) {
        const int row = b * 32 + r;
        const bf16x8 k = *reinterpret_cast<const bf16x8*>(kt + place<kChunks>(row, 2 * t + half));
#pragma unroll
        for (int n = 0; n < kNq; ++n) s[n][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[n][t], s[n][b], 0, 0, 0);
      }
  }

  // Values [4 rows][16 channels] a group of 16 lanes, transposed: this lane's
  // channel 32 d + lane % 32 of rows first .. first + 3 and first + 8 .. first + 11 (first 4 half further).
  __device__ __forceinline__ u32x4 values(const char* vt, int first, int d, int lane) const {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = first + 8 * j + 4 * (lane >> 5) + ((lane >> 2) & 3);
      const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
      const char* at = vt + place<kChunks>(row, chunk) + (lane & 1) * 8;
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
      const u32x2 y = __builtin_bit_cast(u32x2, x);
      w[2 * j] = y[0], w[2 * j + 1] = y[1];
    }
    return w;
  }

  // weights of keys 16 step + ... of block b, as the operand of O^T = V^T P^T; rounded to
  // bfloat16, the type the matrix units take (the sum l is of the unrounded ones)
  __device__ __forceinline__ static bf16x8 weights(const f32x16& s, int step) {
    bf16x8 w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = (__bf16)s[8 * step + j];
    return w;
  }

  // Two values with those that are not finite replaced by zeros.
  __device__ __forceinline__ static uint32_t finite_pair(uint32_t w) {
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu;
    const uint32_t hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
    return lo | hi;
  }

  // With kMasked, values that are not finite enter as zeros (a masked row's
  // weight 0 times NaN or infinity would be NaN); returns whether there were any.
  template <bool kMasked>
  __device__ __forceinline__ uint32_t add_values(const char* vt, int lane, const f32x16 (&s)[kNq][kKeyBlocks]) {
    uint32_t bad = 0;
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 w[kNq];
#pragma unroll
        for (int n = 0; n < kNq; ++n) w[n] = weights(s[n][b], t);
#pragma unroll
        for (int d = 0; d < kOut; ++d) {
          u32x4 raw = values(vt, 32 * b + 16 * t, d, lane);
          if constexpr (kMasked) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t x = finite_pair(raw[j]);
              bad |= raw[j] ^ x;
              raw[j] = x;
            }
          }
          const bf16x8 v = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
          for (int n = 0; n < kNq; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[n], o[n][d], 0, 0, 0);
        }
      }
    return bad;
  }
};

// ---------------------------------------------------------------------------
// float32
// ---------------------------------------------------------------------------
template <int kDim, int kNq, int kKeyBlocks>
struct Core<float, kDim, kNq, kKeyBlocks> {
  static constexpr int kChunks = kDim / 4, kSteps = kDim / 8, kOut = kDim / 32;
  f32x4 q[kNq][kSteps];
  f32x16 o[kNq][kOut];
  float m[kNq], l[kNq];

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < kNq; ++n) {
#pragma unroll
      for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][d][i] = 0.f;
      m[n] = -__builtin_inff();
      l[n] = 0.f;
    }
  }

  __device__ __forceinline__ void load_q(int n, const float* row, int dim, int half) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q[n][s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if ((2 * s + half) * 4 < dim) q[n][s] = *reinterpret_cast<const f32x4*>(row + (2 * s + half) * 4);
    }
  }

  // A lane's chunk holds channels 8 t + 4 half + j: product j of step t takes channels 8 t + j and 8 t + 4 + j.
  __device__ __forceinline__ void scores(const char* kt, int lane, f32x16 (&s)[kNq][kKeyBlocks]) const {
    const int r = lane & 31, half = lane >> 5;
#pragma unroll
    for (int n = 0; n < kNq; ++n)
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][b][i] = 0.f;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b) {
        const int row = b * 32 + r;
        const f32x4 k = *reinterpret_cast<const f32x4*>(kt + place<kChunks>(row, 2 * t + half));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int n = 0; n < kNq; ++n) s[n][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], q[n][t][j], s[n][b], 0, 0, 0);
      }
  }

  // channel 32 d + lane % 32 of key 32 b + 8 (i / 4) + 4 half + i % 4
  __device__ __forceinline__ float value(const char* vt, int b, int i, int d, int lane) const {
    const int row = 32 * b + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
    const int chunk = 8 * d + ((lane & 31) >> 2);
    return *reinterpret_cast<const float*>(vt + place<kChunks>(row, chunk) + (lane & 3) * 4);
  }

  template <bool kMasked>
  __device__ __forceinline__ uint32_t add_values(const char* vt, int lane, const f32x16 (&s)[kNq][kKeyBlocks]) {
    uint32_t bad = 0;
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int d = 0; d < kOut; ++d) {
          float v = value(vt, b, i, d, lane);
          if constexpr (kMasked) {
            const bool fin = finite_f(v);
            bad |= !fin;
            v = fin ? v : 0.f;
          }
#pragma unroll
          for (int n = 0; n < kNq; ++n) o[n][d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[n][b][i], o[n][d], 0, 0, 0);
        }
    return bad;
  }
};

// The values that add_values<true> left out, for the rows that see them: a
// positive weight times NaN or infinity is that value.  Keys [first, end),
// of which kKeys of every kStride are this wave's.
template <class T, class C, int kNq>
__device__ __forceinline__ void add_nonfinite(C& core, const char* base, int64_t stride, int dim, int first, int end, int keys,
                                              int step, const int (&limit)[kNq], int lane) {
  for (int key0 = first; key0 < end; key0 += step)
    for (int key = key0; key < key0 + keys && key < end; ++key) {
      const T* row = (const T*)(base + key * stride);
#pragma unroll
      for (int d = 0; d < C::kOut; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = 32 * d + 8 * g + 4 * (lane >> 5);
          float x[4] = {0.f, 0.f, 0.f, 0.f};
          if (c < dim) load_heads<4>(row + c, x);
#pragma unroll
          for (int n = 0; n < kNq; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) core.o[n][d][4 * g + j] += key < limit[n] && !finite_f(x[j]) ? x[j] : 0.f;
        }
    }
}

// Weights from scores, in place, with the running maximum and sum.  The
// maximum in use follows the true one only where that has grown by more than
// 2^kSlack: the weights stay below 2^kSlack, sums of 2^31 of them stay finite
// in float, and most tiles need no rescaling of the output.
constexpr float kSlack = 8.f;

template <bool kMasked, class C, int kNq, int kKeyBlocks>
__device__ __forceinline__ void softmax_tile(C& core, f32x16 (&s)[kNq][kKeyBlocks], float c, int key0, const int (&limit)[kNq],
                                             int lane) {
#pragma unroll
  for (int n = 0; n < kNq; ++n) {
    if constexpr (kMasked) {
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + 32 * b + 8 * (i / 4) + 4 * (lane >> 5) + i % 4 >= limit[n]) s[n][b][i] = -__builtin_inff();
    }
    float mx = s[n][0][0];
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[n][b][i]);
    mx = max_halves(mx) * c;
    // (row by row, so that a row's rounding does not depend on the others')
    const bool grown = mx > core.m[n] + kSlack;
    if (__any(grown)) {
      const float f = grown ? exp2_hw(core.m[n] - mx) : 1.f;
      if (grown) core.m[n] = mx;
      core.l[n] *= f;
#pragma unroll
      for (int d = 0; d < C::kOut; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) core.o[n][d][i] *= f;
    }
    const float ms = core.m[n] == -__builtin_inff() ? 0.f : core.m[n];
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][b][i] = exp2_hw(__builtin_fmaf(s[n][b][i], c, -ms));
        sum += s[n][b][i];
      }
    core.l[n] += sum;
  }
}

}  // namespace gc
