// Matrix products of few rows: every weight is read once, from memory to registers.
//
// A wave takes 16 weight rows (the first operand; of gates and of values, or 32) 128 bytes of each at a time,
// 32 a lane in two loads, so that the first brings whole lines and the second finds them; eight loads are on their way
// before any is used.  The waves of a block take the same rows' other bytes by turns; their sums
// meet in LDS.  x, read as often as there are blocks, comes from the caches.
// 1 x 6144 x 4096 bfloat16: 11.9 us (4.2 TB/s) with eight waves a block, 12.9 with four; with four, 13.8 past the caches
// and 64 bytes of each row a load, 14.2 with 32 weight rows a wave (from 9 rows of x on 32 are faster).
#pragma once

#include "gc_linear.h"

namespace gc {

// Operands of 16 rows: a 16-byte chunk a lane, row lane % 16.
struct FewF32 {
  __device__ __forceinline__ static f32x4 mma(const u32x4& w, const u32x4& x, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]), c, 0, 0, 0);
    return c;
  }
};
struct FewBF16 {
  __device__ __forceinline__ static f32x4 mma(const u32x4& w, const u32x4& x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
  }
};
struct FewE4M3 {   // as bfloat16, which holds them exactly: there is time for it
  __device__ __forceinline__ static f32x4 mma(const u32x4& w, const u32x4& x, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(E4M3Exact::half(w, i), E4M3Exact::half(x, i), c, 0, 0, 0);
    return c;
  }
};

constexpr int kFewStep = 128;    // bytes of a row that a wave takes at a time
constexpr uint32_t kFewNowhere = 0x7ffffff0u;   // past any range

constexpr int kFewUnroll = 4;    // steps that are read before they are used

// 16 rows of x, 16 weight rows (gated: gates and as many values; wide: 32) and kWaves waves a block.
template <class Op, int kWaves, bool kGated, bool kWide>
__global__ __launch_bounds__(kWaves * 64) void k_linear_few(const LinearArgs p) {
  constexpr int kBlocks = kGated || kWide ? 2 : 1;
  __shared__ f32x4 sums[kWaves][kBlocks][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * (kWide ? 32 : 16);
  const int k_begin = blockIdx.y * p.part_bytes;
  const int k_end = p.row_bytes - k_begin < p.part_bytes ? p.row_bytes : k_begin + p.part_bytes;
  const int rows_x = (int)p.n_rows, rows_w = p.n_out - n0 < 16 ? p.n_out - n0 : 16;
  const int rows_v = !kWide ? rows_w : p.n_out - n0 - 16 < 16 ? p.n_out - n0 - 16 : 16;   // of the second block: none, or fewer
  const int first = lane / 16 * 32;     // byte of the lane's first chunk of a step
  const uint32_t x_at = (uint32_t)(lane % 16) * (uint32_t)p.x_row + first, w_at = (uint32_t)(lane % 16) * (uint32_t)p.w_row + first;
  const char* wb = p.w + (int64_t)n0 * p.w_row;
  const char* vb = wb + (int64_t)(kWide ? 16 : p.n_out) * p.w_row;
  const int range_x = (int)((rows_x - 1) * p.x_row), range_w = (int)((rows_w - 1) * p.w_row);
  const int range_v = (int)((rows_v - 1) * p.w_row);

  f32x4 acc[kBlocks];
#pragma unroll
  for (int j = 0; j < kBlocks; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = k_begin + wave * kFewStep * kFewUnroll; k < k_end; k += kWaves * kFewStep * kFewUnroll) {
    u32x4 w[2 * kFewUnroll][kBlocks], x[2 * kFewUnroll];
#pragma unroll
    for (int u = 0; u < 2 * kFewUnroll; ++u) {
      const int at = k + u / 2 * kFewStep, left = k_end - at;
      // past the end of a row, and past the last row, zeros arrive
      const bool past = first + u % 2 * 16 >= left;
      const uint32_t from_w = past ? kFewNowhere : w_at + u % 2 * 16, from_x = past ? kFewNowhere : x_at + u % 2 * 16;
      const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)(wb + at), 0, left > 0 ? range_w + left : 0, 0x00027000);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(vb + at), 0, left > 0 && rows_v > 0 ? range_v + left : 0, 0x00027000);
      const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)(p.x + at), 0, left > 0 ? range_x + left : 0, 0x00027000);
      w[u][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, from_w, 0, 0));
      if (kBlocks == 2) w[u][kBlocks - 1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rv, from_w, 0, 0));
      x[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, from_x, 0, 0));
    }
    __builtin_amdgcn_sched_barrier(0);   // all reads before any use
#pragma unroll
    for (int u = 0; u < 2 * kFewUnroll; ++u)
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) acc[j] = Op::mma(w[u][j], x[u], acc[j]);
  }
  // one output a thread: row m of x and weight row n
  const int n = threadIdx.x % 16, m = kWide ? threadIdx.x / 16 % 16 : threadIdx.x / 16, second = kWide ? threadIdx.x / 256 : 0;
  const int col = n0 + 16 * second + n;
  const bool mine = m < rows_x && second < 2 && col < p.n_out;
  Column c;
  OneAhead row;
  if (mine && p.parts == 1) c.init<kGated>(p, col), row.load(p, m, col);
#pragma unroll
  for (int j = 0; j < kBlocks; ++j) sums[wave][j][lane] = acc[j];
  __syncthreads();

  // they are lane n / 4 * 16 + m of a block's sums, element n % 4
  if (!mine) return;
  const int from = n / 4 * 16 + m;
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    a += sums[v][kWide ? second : 0][from][n % 4];
    if (kGated) b += sums[v][kBlocks - 1][from][n % 4];
  }
  if (p.parts > 1) {
    float* o = p.partial + blockIdx.y * p.partial_part + (int64_t)m * p.partial_cols * (kGated ? 2 : 1) + col;
    o[0] = a;
    if (kGated) o[p.partial_cols] = b;
  } else {
    finish_one<kGated>(p, c, m, row, a, b);
  }
}

}  // namespace gc
