// Matrix products in tiles: a block computes kX rows by kW rows of the weights.
//
// Both operands are rows with the inner dimension contiguous, so either tile is
// read from memory to LDS 128 bytes of each row at a time, straight and
// 16 bytes a lane, with chunk c of row r at place c ^ (r / 2 % 8): then
// 16 rows' same chunk lie in 16 different places of the 256 bytes that the banks span.
//
// The weights are the first operand, so an accumulator's lane holds one row of
// x and 16 weight rows.  Which weight row lies at which place of a 32-row
// block is free: row 8 a + 4 h + b of the product is weight row 16 h + 4 a + b, so that
// a lane's 16 outputs are consecutive.  Gated products take blocks of 32 gate and 32 value rows by
// turns, so that a lane holds both.
#pragma once

#include "gc_linear.h"

namespace gc {

typedef __attribute__((address_space(3))) void LdsVoid;

template <int kLeft>
__device__ __forceinline__ void wait_for_loads() {
  static_assert(kLeft < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | (7 << 4) | (15 << 8) | ((kLeft >> 4) << 14));
  asm volatile("" ::: "memory");
}

constexpr int kStepBytes = 128;   // of a row, a step

__device__ __forceinline__ int tile_place(int row, int chunk) { return row * kStepBytes + ((chunk ^ (row >> 1)) & 7) * 16; }

template <class Op, int kWavesX, int kWavesW, int kBlocksX, int kBlocksW, bool kGated>
struct Tiles {
  static constexpr int kWaves = kWavesX * kWavesW, kThreads = kWaves * 64;
  static constexpr int kX = kWavesX * kBlocksX * 32, kW = kWavesW * kBlocksW * 32;
  static constexpr int kOut = kGated ? kW / 2 : kW;      // columns of the output
  static constexpr int kStage = (kX + kW) * kStepBytes;
  static constexpr int kLoads = (kX + kW) / 8 / kWaves;  // a wave's, a step
  static_assert((kX + kW) / 8 % kWaves == 0 && kX / 8 % kWaves == 0 && kWaves % 4 == 0, "whole loads");
  static_assert(!kGated || kBlocksW % 2 == 0, "gate and value in one wave");
};

template <class Op, int kWavesX, int kWavesW, int kBlocksX, int kBlocksW, bool kGated>
__global__ __launch_bounds__(kWavesX* kWavesW * 64) void k_linear_tiles(const LinearArgs p) {
  using C = Tiles<Op, kWavesX, kWavesW, kBlocksX, kBlocksW, kGated>;
  extern __shared__ char lds[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = (int64_t)blockIdx.y * C::kX;
  const int n0 = blockIdx.x * C::kOut;

  // the rows that this lane's loads read, and their chunk
  const int chunk = (lane ^ (lane >> 4) ^ (wave << 2)) & 7;   // rows of a load: 8 (wave + ..) + lane / 8
  const int left_x = p.n_rows - m0 < C::kX ? (int)(p.n_rows - m0) : C::kX;
  const int left_w = p.n_out - n0;
  const int k_begin = 0, k_end = p.row_bytes;
  uint32_t at[C::kLoads];
#pragma unroll
  for (int i = 0; i < C::kLoads; ++i) {
    const int row = 8 * (wave + i * C::kWaves) + (lane >> 3);
    if (8 * (wave + i * C::kWaves) < C::kX) {
      at[i] = (uint32_t)row * (uint32_t)p.x_row + chunk * 16;
    } else {
      const int r = row - C::kX, block = r >> 5, in = ((r >> 2) & 1) * 16 + ((r >> 3) & 3) * 4 + (r & 3);
      at[i] = (uint32_t)((kGated ? block >> 1 : block) * 32 + in) * (uint32_t)p.w_row + chunk * 16;
    }
  }
  const int rows_w = left_w < C::kOut ? left_w : C::kOut;

  f32x16 acc[kBlocksX][kBlocksW];
#pragma unroll
  for (int i = 0; i < kBlocksX; ++i)
#pragma unroll
    for (int j = 0; j < kBlocksW; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  const int wx = wave / kWavesW, ww = wave % kWavesW;
  for (int k = k_begin; k < k_end; k += kStepBytes) {
    const int left = k_end - k;
    const bool past = chunk * 16 >= left;
    const char* xb = p.x + m0 * p.x_row + k;
    const char* wb = p.w + (int64_t)n0 * p.w_row + k;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)xb, 0, (int)((left_x - 1) * p.x_row) + left, 0x00027000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)wb, 0, (int)((rows_w - 1) * p.w_row) + left, 0x00027000);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(wb + (int64_t)p.n_out * p.w_row), 0, (int)((rows_w - 1) * p.w_row) + left, 0x00027000);
#pragma unroll
    for (int i = 0; i < C::kLoads; ++i) {
      const int first = 8 * (wave + i * C::kWaves);
      const bool of_x = first < C::kX;
      const bool value = kGated && !of_x && (((first - C::kX) >> 5) & 1);
      LdsVoid* to = (LdsVoid*)(lds + first * kStepBytes);
      const uint32_t from = past ? 0x7ffffff0u : at[i];
      if (of_x) __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, to, 16, from, 0, 0, 0);
      else if (value) __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, to, 16, from, 0, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, to, 16, from, 0, 0, 0);
    }
    wait_for_loads<0>();
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 4 / Op::kPairs; ++s) {
      typename Op::Frag x[kBlocksX], w[kBlocksW];
#pragma unroll
      for (int i = 0; i < kBlocksX; ++i) {
        u32x4 c[Op::kPairs];
#pragma unroll
        for (int q = 0; q < Op::kPairs; ++q)
          c[q] = *reinterpret_cast<const u32x4*>(lds + tile_place((wx * kBlocksX + i) * 32 + (lane & 31), 2 * (s * Op::kPairs + q) + (lane >> 5)));
        __builtin_memcpy(&x[i], c, sizeof(x[i]));
      }
#pragma unroll
      for (int j = 0; j < kBlocksW; ++j) {
        u32x4 c[Op::kPairs];
#pragma unroll
        for (int q = 0; q < Op::kPairs; ++q)
          c[q] = *reinterpret_cast<const u32x4*>(lds + tile_place(C::kX + (ww * kBlocksW + j) * 32 + (lane & 31), 2 * (s * Op::kPairs + q) + (lane >> 5)));
        __builtin_memcpy(&w[j], c, sizeof(w[j]));
      }
#pragma unroll
      for (int i = 0; i < kBlocksX; ++i)
#pragma unroll
        for (int j = 0; j < kBlocksW; ++j) acc[i][j] = Op::mma(w[j], x[i], acc[i][j]);
    }
    __syncthreads();
  }

#pragma unroll
  for (int i = 0; i < kBlocksX; ++i)
#pragma unroll
    for (int j = 0; j < kBlocksW; j += kGated ? 2 : 1) {
      const int64_t m = m0 + (wx * kBlocksX + i) * 32 + (lane & 31);
      const int n = n0 + (ww * kBlocksW + j) * (kGated ? 16 : 32) + (lane >> 5) * 16;
      float a[16], b[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) a[e] = acc[i][j][e], b[e] = kGated ? acc[i][j + (kGated ? 1 : 0)][e] : 0.f;
      finish<16>(p, m, n, a, b);
    }
}

}  // namespace gc
