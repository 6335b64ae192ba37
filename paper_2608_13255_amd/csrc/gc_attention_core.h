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
// Why 32 x 32 blocks: an operand read from LDS feeds 32 x 32 x 16 products,
// half the LDS traffic of 16 x 16 blocks; with 32 rows a wave of bfloat16
// holds 64 keys' scores twice beside the output of up to 128 channels within
// the 256 registers of two waves a SIMD.  64 rows a wave would halve the LDS reads
// again but spill (8.8 ms where 32 rows took 4.3).  Above 128 channels a SIMD
// has one wave, and nothing runs beside its vector work.  In float32 its 512
// registers do not hold everything there: 348 and 632 bytes a lane of a
// prompt's kernel lie in scratch at 192 and 256, 216 of a single token's at
// 256 (bfloat16: 8 at 128 channels with eight waves, outside the loop over whole tiles).
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
  int kv_heads, group, dim;
  int total_q;
  int causal;
  float scale;
  float* partial;       // per slot and kv head: [tile_rows][dim padded] weighted sums, then [tile_rows][2] maxima and sums
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
// The factor of a weighted sum whose maximum falls behind by x (in powers of two): never 0, which would make NaN of a
// sum of infinity.
__device__ __forceinline__ float sum_factor(float x) { return fmaxf(exp2_hw(x), 0x1p-149f); }

// The larger of a lane's value and that of the lane 32 away; their sum.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Copies tiles of kKeys rows of a K or V tensor, one after the other, to LDS
// with the permutation, straight from memory (buffer loads to LDS: 16 bytes a
// lane, places in lane order).  Rows past the last key, and channels past
// dim, arrive as zeros: the buffer's range ends there.  Tiles are kStep tiles
// apart.  kOnce: rows that no other block reads, past the caches (single
// tokens over 495 MB of keys and values: 89 us against 103).
template <class T, int kDim, int kKeys, int kWaves, int kStep = 1, bool kOnce = false>
struct TileLoader {
  static constexpr int kChunks = kDim * (int)sizeof(T) / 16;
  static constexpr int kLoads = kKeys * kChunks / 64;     // of a wave's 64 lanes
  static constexpr int kMine = (kLoads + kWaves - 1) / kWaves;
  static_assert(kKeys * kChunks % 64 == 0, "whole loads");
  const char* at;         // the next tile's first row
  int64_t advance;        // bytes to the one after
  int left;               // keys from there to the end
  int stride, row_bytes;
  uint32_t offset[kMine];

  // keys [first, end) of a sequence that starts at first_token
  __device__ __forceinline__ void init(const void* p, int64_t first_token, int64_t token_stride, int64_t head_off, int dim,
                                       int first, int end, int wave, int lane) {
    const int64_t bytes = token_stride * (int64_t)sizeof(T);
    at = (const char*)p + (first_token + first) * bytes + head_off * (int64_t)sizeof(T);
    advance = bytes * (kKeys * kStep);
    left = end - first;
    stride = (int)bytes;
    row_bytes = dim * (int)sizeof(T);
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const int place16 = (wave + n * kWaves) % kLoads * 64 + lane;
      // the chunk that lies at this place: the exclusive or is its own inverse
      const int row = place16 / kChunks, chunk = place<kChunks>(row, place16 % kChunks) / 16 - row * kChunks;
      offset[n] = chunk * 16 < row_bytes ? (uint32_t)row * (uint32_t)stride + (uint32_t)chunk * 16u : 0x7ffffff0u;
    }
  }

  // The next tile.  Past the end nothing is read (and the places get zeros): the number of loads outstanding is the same.
  __device__ __forceinline__ void load(char* lds, int wave) {
    const int rows = left < kKeys ? left : kKeys, some = (rows - 1) * stride + row_bytes;
    const int bytes = rows > 0 ? some : 0;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, bytes, 0x00027000);
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      // (where the loads are no multiple of the waves, some are made twice: every wave has the same number outstanding)
      const int i = (wave + n * kWaves) % kLoads;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid*)(lds + i * 1024), 16, offset[n], 0, 0, kOnce ? 2 : 0);
    }
    at += advance;
    left -= kKeys * kStep;
  }
};

// Until at most kLeft of the wave's loads are outstanding.
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  static_assert(kLeft < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | (7 << 4) | (15 << 8) | ((kLeft >> 4) << 14));
  asm volatile("" ::: "memory");
}

// A query row: its token, head and the keys that it sees.
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
// What one wave holds: the queries of 32 rows (an operand of
// S^T), O^T, and the rows' maximum in use and sum.  A tile is kKeyBlocks * 32
// keys.
template <class T, int kDim, int kKeyBlocks>
struct Core;

// S^T: key 32 b + 8 (i / 4) + 4 half + i % 4
template <int kKeyBlocks>
struct Scores {
  f32x16 s[kKeyBlocks];
};

template <int kOut>
struct Accumulators {
  f32x16 o[kOut];
  float m, l;   // maximum in use (score times scale times log2 e) and this lane's part of the sum
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    m = -__builtin_inff();
    l = 0.f;
  }
};

template <int kDim, int kKeyBlocks>
struct Core<uint16_t, kDim, kKeyBlocks> : Accumulators<kDim / 32> {
  static constexpr int kChunks = kDim / 8, kSteps = kDim / 16, kOut = kDim / 32;
  // operands of the scores and of the output, a product each
  static constexpr int kOperands = kKeyBlocks * kSteps, kAhead = kOperands < 4 ? kOperands : 4;
  static_assert(kOperands == 2 * kKeyBlocks * kOut, "as many of either kind");
  using Accumulators<kOut>::o;
  using Accumulators<kOut>::l;
  using S = Scores<kKeyBlocks>;
  bf16x8 q[kSteps];

  // Weights as an operand of O^T = V^T P^T: element j of group g is key 16 g + 8 (j / 4) + 4 half + j % 4.  Rounded to
  // bfloat16, the type that the matrix units take; the sum l is of the unrounded ones.  The error of a
  // prompt's output against 64 bits is 0.0024 in the 2-norm with it, where rounding the output alone gives 0.0017.
  struct Weights {
    bf16x8 w[2 * kKeyBlocks];
  };

  __device__ __forceinline__ void load_q(const uint16_t* row, int dim, int half) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if ((2 * s + half) * 8 < dim) w = *reinterpret_cast<const u32x4*>(row + (2 * s + half) * 8);
      q[s] = __builtin_bit_cast(bf16x8, w);
    }
  }

  // Operand i of the scores: key block i % kKeyBlocks, channels 16 (i / kKeyBlocks) + 8 half ..
  __device__ __forceinline__ static bf16x8 keys(const char* kt, int lane, int i) {
    const int row = i % kKeyBlocks * 32 + (lane & 31);
    return *reinterpret_cast<const bf16x8*>(kt + place<kChunks>(row, 2 * (i / kKeyBlocks) + (lane >> 5)));
  }
  __device__ __forceinline__ void score(S& s, bf16x8 k, int i) const {
      s.s[i % kKeyBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[i / kKeyBlocks], s.s[i % kKeyBlocks], 0, 0, 0);
  }
  __device__ __forceinline__ static void clear(S& s) {
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s.s[b][i] = 0.f;
  }
  __device__ __forceinline__ void scores(const char* kt, int lane, S& s) const {
    clear(s);
#pragma unroll
    for (int i = 0; i < kOperands; ++i) score(s, keys(kt, lane, i), i);
  }

  // Operand i of the output: group i / kOut of the weights' keys, channels 32 (i % kOut) + lane % 32.  Two reads that
  // transpose: four rows of 16 channels a group of 16 lanes, from rows first .. first + 3 and first + 8 .. first + 11
  // (first 4 half further).  A lane's places in the first group are kept in registers, since the permutation hides from
  // the compiler that the other groups' are whole rows further (with places computed where they are needed the
  // reads came late: 10403 tokens in four sequences x 16 heads x 64 152 us).
  int value_at[2][kOut];
  __device__ __forceinline__ void init_values(int lane) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int d = 0; d < kOut; ++d) {
        const int row = 8 * j + 4 * (lane >> 5) + ((lane >> 2) & 3);
        const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        value_at[j][d] = place<kChunks>(row, chunk) + (lane & 1) * 8;
        asm volatile("" : "+v"(value_at[j][d]));
      }
  }
  __device__ __forceinline__ u32x4 values(const char* vt, int i) const {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const char* at = vt + value_at[j][i % kOut] + i / kOut * (16 * kChunks * 16);
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
      const u32x2 y = __builtin_bit_cast(u32x2, x);
      w[2 * j] = y[0], w[2 * j + 1] = y[1];
    }
    return w;
  }
  __device__ __forceinline__ void add(const Weights& w, u32x4 v, int i) {
      o[i % kOut] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), w.w[i / kOut], o[i % kOut], 0, 0, 0);
  }

  // Two values with those that are not finite replaced by zeros.
  __device__ __forceinline__ static uint32_t finite_pair(uint32_t w) {
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu;
    const uint32_t hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
    return lo | hi;
  }

  // A tile's values, where rows may be masked: those that are not finite enter as zeros (a masked row's weight 0 times NaN
  // or infinity would be NaN).  Returns whether there were any (add_nonfinite).  The largest magnitude, as an
  // integer, tells of a few operands at a time whether one is to be replaced (two instructions a pair of values
  // against ten: 4096 causal tokens x 8 heads x 128 53.8 us against 56.9).
  __device__ __forceinline__ uint32_t add_masked(const char* vt, int, const Weights& w) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    constexpr int kGroup = kOperands % 4 == 0 ? 4 : 2;
    uint32_t bad = 0;
#pragma unroll
    for (int i0 = 0; i0 < kOperands; i0 += kGroup) {
      u32x4 v[kGroup];
#pragma unroll
      for (int i = 0; i < kGroup; ++i) v[i] = values(vt, i0 + i);
      u16x2 top = {0, 0};
#pragma unroll
      for (int i = 0; i < kGroup; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[i][j] & 0x7fff7fffu));
      if (__any(top[0] >= 0x7f80 || top[1] >= 0x7f80)) {
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t x = finite_pair(v[i][j]);
            bad |= v[i][j] ^ x;
            v[i][j] = x;
          }
      }
#pragma unroll
      for (int i = 0; i < kGroup; ++i) add(w, v[i], i0 + i);
    }
    return bad;
  }
  __device__ __forceinline__ void add_values(const char* vt, int, const Weights& w) {
#pragma unroll
    for (int i = 0; i < kOperands; ++i) add(w, values(vt, i), i);
  }

  __device__ __forceinline__ void weight(const S& s, float c, float ms, Weights& w, int e, float& sum) const {
    const float x = exp2_hw(__builtin_fmaf(s.s[e / 16][e % 16], c, -ms));
    sum += x;
    w.w[e / 8][e % 8] = (__bf16)x;
  }
  __device__ __forceinline__ void weights(const S& s, float c, float ms, Weights& w) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16 * kKeyBlocks; ++e) weight(s, c, ms, w, e, sum);
    l += sum;
  }

  // The two parts of a tile's work when nothing is masked.  Each runs matrix
  // products beside vector work that does not need them: a wave issues a few
  // vector instructions while a product runs.  A part asks for its operands
  // kAhead products ahead, and for the first ones of the part after it.
  struct Operands {
    bf16x8 k[kAhead];
    u32x4 v[kAhead];
  };
  __device__ __forceinline__ void first_values(const char* vt, Operands& x) const {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x.v[i] = values(vt, i);
  }

  // the values of the tile before, and this tile's largest scores (of this lane's)
  __device__ __forceinline__ void values_and_maximum(Operands& x, const char* vt, const Weights& w, const S& s, const char* kt,
                                                     int lane, float& mx) {
    u32x4 v[kOperands];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = x.v[i];
    constexpr int kPairs = 8 * kKeyBlocks;   // of scores
    mx = s.s[0][0];
#pragma unroll
    for (int i = 0; i < kOperands; ++i) {
      if (i + kAhead < kOperands) v[i + kAhead] = values(vt, i + kAhead);
      else x.k[i + kAhead - kOperands] = keys(kt, lane, i + kAhead - kOperands);
      add(w, v[i], i);
#pragma unroll
      for (int e = i * kPairs / kOperands; e < (i + 1) * kPairs / kOperands; ++e) {
        const int y = 2 * e;
        mx = fmaxf(fmaxf(mx, s.s[y / 16][y % 16]), s.s[y / 16][y % 16 + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < kOperands; ++i) {
      if (i + kAhead < kOperands) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      else __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, (8 * kKeyBlocks + kOperands - 1) / kOperands, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // this tile's weights, and the next tile's scores
  __device__ __forceinline__ void weights_and_scores(Operands& x, const S& s, float c, float ms, Weights& w,
                                                     const char* kt, S& next, const char* vt, int lane) {
    bf16x8 k[kOperands];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) k[i] = x.k[i];
    constexpr int kWeights = 16 * kKeyBlocks;
    float sum = 0.f;
    clear(next);
#pragma unroll
    for (int i = 0; i < kOperands; ++i) {
      if (i + kAhead < kOperands) k[i + kAhead] = keys(kt, lane, i + kAhead);
      else x.v[i + kAhead - kOperands] = values(vt, i + kAhead - kOperands);
      score(next, k[i], i);
#pragma unroll
      for (int e = i * kWeights / kOperands; e < (i + 1) * kWeights / kOperands; ++e)
        weight(s, c, ms, w, e, sum);
    }
    l += sum;
    // here and not where they are used, in the next part
#pragma unroll
    for (int g = 0; g < 2 * kKeyBlocks; ++g) asm volatile("" : "+v"(w.w[g]));
#pragma unroll
    for (int i = 0; i < kOperands; ++i) {
      if (i + kAhead < kOperands) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      else __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 7 * 8 * kKeyBlocks / kOperands, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
};

// ---------------------------------------------------------------------------
// float32
// ---------------------------------------------------------------------------
template <int kDim, int kKeyBlocks>
struct Core<float, kDim, kKeyBlocks> : Accumulators<kDim / 32> {
  static constexpr int kChunks = kDim / 4, kSteps = kDim / 8, kOut = kDim / 32;
  using Accumulators<kOut>::o;
  using Accumulators<kOut>::l;
  using S = Scores<kKeyBlocks>;
  f32x4 q[kSteps];

  struct Weights {
    f32x16 w[kKeyBlocks];   // in the scores' order, a key a product
  };

  __device__ __forceinline__ void load_q(const float* row, int dim, int half) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q[s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if ((2 * s + half) * 4 < dim) q[s] = *reinterpret_cast<const f32x4*>(row + (2 * s + half) * 4);
    }
  }

  // A lane's chunk holds channels 8 t + 4 half + j: product j of step t takes channels 8 t + j and 8 t + 4 + j.
  __device__ __forceinline__ void scores(const char* kt, int lane, S& s) const {
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s.s[b][i] = 0.f;
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int b = 0; b < kKeyBlocks; ++b) {
        const f32x4 k = *reinterpret_cast<const f32x4*>(kt + place<kChunks>(b * 32 + (lane & 31), 2 * t + (lane >> 5)));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s.s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[j], q[t][j], s.s[b], 0, 0, 0);
      }
  }

  __device__ __forceinline__ void weights(const S& s, float c, float ms, Weights& w) {
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w.w[b][i] = exp2_hw(__builtin_fmaf(s.s[b][i], c, -ms));
        sum += w.w[b][i];
      }
    l += sum;
  }

  __device__ __forceinline__ void init_values(int) {}
  // channel 32 d + lane % 32 of key 32 b + 8 (i / 4) + 4 half + i % 4
  __device__ __forceinline__ static float value(const char* vt, int b, int i, int d, int lane) {
    const int row = 32 * b + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
    const int chunk = 8 * d + ((lane & 31) >> 2);
    return *reinterpret_cast<const float*>(vt + place<kChunks>(row, chunk) + (lane & 3) * 4);
  }

  template <bool kMasked>
  __device__ __forceinline__ uint32_t add_all(const char* vt, int lane, const Weights& w) {
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
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w.w[b][i], o[d], 0, 0, 0);
        }
    return bad;
  }
  __device__ __forceinline__ uint32_t add_masked(const char* vt, int lane, const Weights& w) { return add_all<true>(vt, lane, w); }
  __device__ __forceinline__ void add_values(const char* vt, int lane, const Weights& w) { add_all<false>(vt, lane, w); }
};

// The values that add_masked left out, for the rows that see them: a
// positive weight times NaN or infinity is that value.  Keys [first, end),
// of which `keys` of every `step` are this wave's.
template <class T, class C>
__device__ __forceinline__ void add_nonfinite(const AttentionArgs& p, const AttentionItem& it, int kv_head, C& core, int first,
                                              int end, int keys, int step, int limit, int lane) {
  for (int key0 = first; key0 < end; key0 += step)
    for (int key = key0; key < key0 + keys && key < end; ++key) {
      const T* row = (const T*)p.v + ((int64_t)it.k_token0 + key) * p.v_token + kv_head * p.v_head;
#pragma unroll
      for (int d = 0; d < C::kOut; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = 32 * d + 8 * g + 4 * (lane >> 5);
          float x[4] = {0.f, 0.f, 0.f, 0.f};
          if (c < p.dim) load_heads<4>(row + c, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) core.o[d][4 * g + j] += key < limit && !finite_f(x[j]) ? x[j] : 0.f;
        }
    }
}

// Whether one of a lane's sums is not finite: 0 times any of them is 0 else.
template <class C>
__device__ __forceinline__ bool any_nonfinite(const C& core) {
  float x = 0.f;
#pragma unroll
  for (int d = 0; d < C::kOut; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x = __builtin_fmaf(core.o[d][i], 0.f, x);
  return x != x;
}

// Values that are not finite leave infinity or NaN in their channel: NaN also
// where a row's weight, against the maximum in use at the time, underflowed to
// 0.  A row's channel is to hold the sum of such values that it sees, however
// small their weights, so the channels that are NaN are looked up again.  Not
// where l is NaN: the row's scores are.
// Keys [first, end), of which `keys` (at most 64) of every `step` are this
// wave's; each lane looks at one of them, the last ones first (the masked
// tiles' have just been added).
template <class T, class C>
__device__ __forceinline__ void settle_nonfinite(const AttentionArgs& p, const AttentionItem& it, int kv_head, C& core, float l,
                                                 int first, int end, int keys, int step, int limit, int lane) {
  const auto is_nan = [](float x) { return x != x; };
  if (first >= end || __builtin_expect(!__any(any_nonfinite(core) && !is_nan(l)), 1)) return;
  const T* values = (const T*)p.v + (int64_t)it.k_token0 * p.v_token + kv_head * p.v_head;
  for (int n = 0; 8 * n < p.dim; ++n) {   // channels 8 n .. 8 n + 7, the lane's own from 8 n + 4 half
    float o[4];
#pragma unroll
    for (int i = 0; i < 4 * C::kOut; ++i)
      if (i == n)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = core.o[i / 4][i % 4 * 4 + j];
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t hit = 0;
    const auto open = [&] {
      bool x = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) x |= is_nan(o[j]) && !is_nan(sum[j]);
      return __any(x && !is_nan(l)) != 0;
    };
    for (int key0 = first + (end - 1 - first) / step * step; key0 >= first && open(); key0 -= step) {
      const int mine = key0 + lane;
      bool some = false;
      if (lane < keys && mine < end) {
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          float x[4];
          load_heads<4>(values + (int64_t)mine * p.v_token + 8 * n + j, x);
          some |= !(finite_f(x[0]) && finite_f(x[1]) && finite_f(x[2]) && finite_f(x[3]));
        }
      }
      for (uint64_t left = __ballot(some); left; left &= left - 1) {
        const int key = key0 + __builtin_ctzll(left);
        float x[4];
        load_heads<4>(values + (int64_t)key * p.v_token + 8 * n + 4 * (lane >> 5), x);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (key < limit && !finite_f(x[j])) sum[j] += x[j], hit |= 1u << j;
      }
    }
#pragma unroll
    for (int i = 0; i < 4 * C::kOut; ++i)
      if (i == n)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (is_nan(o[j]) && (hit >> j & 1)) core.o[i / 4][i % 4 * 4 + j] = sum[j];
  }
  // (else the compiler waits for these loads, and so for earlier stores, between the stores of the results)
  wait_loads<0>();
}

// Masked places' scores.
template <int kKeyBlocks>
__device__ __forceinline__ void mask(Scores<kKeyBlocks>& s, int key0, int limit, int lane) {
#pragma unroll
    for (int b = 0; b < kKeyBlocks; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (key0 + 32 * b + 8 * (i / 4) + 4 * (lane >> 5) + i % 4 >= limit) s.s[b][i] = -__builtin_inff();
}

template <int kKeyBlocks>
__device__ __forceinline__ void maximum(const Scores<kKeyBlocks>& s, float& mx) {
  mx = s.s[0][0];
#pragma unroll
  for (int e = 1; e < 16 * kKeyBlocks; ++e) mx = fmaxf(mx, s.s[e / 16][e % 16]);
}

// The running maximum.  The one in use follows the true one only where that
// has grown by more than kSlack (in powers of two): the weights stay far
// below float's range, and most tiles need no rescaling of the output.  Row
// by row, so that a row's rounding does not depend on the others'.
constexpr float kSlack = 8.f;

template <class C>
__device__ __forceinline__ void rescale(C& core, bool grown, float top) {
  const float f = grown ? sum_factor(core.m - top) : 1.f;
  if (grown) core.m = top;
  core.l *= f;
#pragma unroll
  for (int d = 0; d < C::kOut; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) core.o[d][i] *= f;
}

// With a tile's largest score mx (a lane's own); ms: what the weights' exponents are taken against.
template <class C>
__device__ __forceinline__ void update_maximum(C& core, float mx, float c, float& ms) {
  const float top = max_halves(mx) * c;
  const bool grown = top > core.m + kSlack;
  if (__any(grown)) rescale(core, grown, top);
  ms = core.m == -__builtin_inff() ? 0.f : core.m;
}

}  // namespace gc
