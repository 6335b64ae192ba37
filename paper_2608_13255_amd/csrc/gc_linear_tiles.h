// Matrix products in tiles: a block computes kX rows by kW rows of the weights.
//
// Both operands are rows with the inner dimension contiguous, so either tile is
// read from memory to LDS 128 bytes of each row at a time (a step), straight and
// 16 bytes a lane, with chunk c of row r at place c ^ (r / 2 % 8): then
// 16 rows' same chunk lie in 16 different places of the 256 bytes that the banks span.
// kBuffers steps are in LDS or on their way: when every wave has read a step, its place is filled again.
//
// The weights are the first operand, so an accumulator's lane holds one row of
// x and groups of four consecutive weight rows.  Gated products take 32 gate and 32 value rows by
// turns, so that a wave holds both.
//
// What bounds it: power and the steps' arrival.  8192^3 bfloat16: 759 us (1450 TFLOP/s), matrix units busy 75 % of the time at
// 1.78 GHz; without the loads of the steps 671, without the epilogue 719.  The library takes 673.  What counted there:
//   products of 16 x 16 instead of 32 x 32 (791 and 845; float32, 2048^3: 128 and 135), with less power; eight waves (828 with four of 128 x 128)
//   a step's loads all at once after the barrier that frees their place (789 spread over the step)
//   lines asked for half a step before their loads, by one of the blocks that share them (852 without)
//   128 bytes of a row a load: with 64 bytes and four steps on their way the L2 gets twice the requests (866)
// Blocks that stay and take tiles by turns were slower (24576 x 16384 x 4096 2590, 2497): all units then
// write at the same time, and wait for it.
#pragma once

#include "gc_linear.h"

namespace gc {

typedef __attribute__((address_space(3))) void LdsVoid;

// Until at most kLeft of the wave's loads from memory are outstanding, and none of its reads of LDS.
template <int kLeft>
__device__ __forceinline__ void wait_all_but() {
  static_assert(kLeft < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | (7 << 4) | (0 << 8) | ((kLeft >> 4) << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

constexpr int kTotalSteps = 16;
constexpr uint32_t kNowhere = 0x7ffffff0u;   // past any range
// Blocks that share rows of x, or of the weights, and the steps between a line asked for and the one to be loaded next.
constexpr int kAheadW = 4, kAheadX = 8, kAheadSteps = 0;

template <class Op_, int kWavesX_, int kWavesW_, int kRowsX, int kRowsW, int kBuffers_, bool kGated_>
struct Tiles {
  typedef Op_ Op;
  static constexpr int kWavesX = kWavesX_, kWavesW = kWavesW_;
  static constexpr bool kGated = kGated_, kTotals = Op::kTotals;
  static constexpr int kWaves = kWavesX * kWavesW, kThreads = kWaves * 64;
  static constexpr int kBlocksX = kRowsX / Op::kBlock, kBlocksW = kRowsW / Op::kBlock;   // of a wave
  static constexpr int kX = kWavesX * kRowsX, kW = kWavesW * kRowsW;
  static constexpr int kWaveX = kRowsX, kWaveW = kRowsW;
  static constexpr int kOut = kGated ? kW / 2 : kW;      // columns of the output
  static constexpr int kBuffers = kBuffers_;
  static constexpr int kStage = (kX + kW) * kStepBytes;
  static constexpr int kLoads = (kX + kW) / 8 / kWaves;      // a wave's, a step
  static constexpr int kGroups = 64 / Op::kBlock;            // of lanes
  static constexpr int kParts = 8 / kGroups / Op::kChunks;   // of a step: fragments that products take
  static constexpr int kFrags = kBlocksX + kBlocksW;
  static constexpr int kLds = kBuffers * kStage + kWaves * 256;
  // the epilogue's place of a wave, where the steps lay: its sums, or a half or third of their rows
  static constexpr int kPlace = kBuffers * kStage / kWaves;
  static constexpr bool fits(int passes) { return kRowsX % ((kRowsX < 32 ? 16 : 32) * passes) == 0 && kRowsX / passes * kRowsW * 4 <= kPlace; }
  static constexpr int kPasses = fits(1) ? 1 : fits(2) ? 2 : 3, kPassRows = kRowsX / kPasses;
  static constexpr int kWaveFloats = kPassRows * kRowsW;
  // A round of large tiles writes what all L2s hold, at once: past the caches (24576 x 16384 x 1024 bfloat16, a result of 805
  // MB, 763 us, 817 through them).  By the tile alone: a result of tens of MB that is read at once was not timed with its reader.
  static constexpr bool kOnce = kX * kW >= 192 * 256;
  static constexpr int kAtOnce = 163840 / kLds;   // blocks on a compute unit
  static_assert(fits(kPasses), "room for the epilogue");
  static_assert(kLds <= 163840 && (kRowsW == 64 || kRowsW == 32), "LDS of a compute unit, and what the epilogue's permutation covers");
  static_assert((kX + kW) / 8 % kWaves == 0 && kX / 8 % kWaves == 0 && kWaves % 4 == 0, "whole loads");
  static_assert(!kGated || kRowsW % 64 == 0, "gate and value in one wave");
};

// Tiles and parts of the inner dimension, as blocks take them: consecutive blocks go to the eight XCDs by turns, each
// with an L2 of its own, so each XCD has a run of tiles, and walks it kGroup tiles of x high.
struct TileAt {
  int x, w, part;
};
__device__ __forceinline__ TileAt tile_at(int id, int tiles_x, int tiles_w, int parts) {
  constexpr int kXcds = 8, kGroup = 8;
  const int tiles = tiles_x * tiles_w, n = tiles * parts, q = n / kXcds, r = n % kXcds;
  const int xcd = id % kXcds, all = xcd * q + (xcd < r ? xcd : r) + id / kXcds;
  const int part = all / tiles, at = all - part * tiles;
  const int group = at / (kGroup * tiles_w), first = group * kGroup;
  const int high = tiles_x - first < kGroup ? tiles_x - first : kGroup;
  const int in = at - group * kGroup * tiles_w;
  return {first + in % high, in / high, part};
}

// The lane's number, where nothing computed from it before is kept in registers until here.
__device__ __forceinline__ int lane_anew() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}

// The kernel's arguments, read again here: kept in scalar registers from the start they would not leave enough of them.
__device__ __forceinline__ LinearArgs args_anew() {
  typedef const __attribute__((address_space(4))) uint64_t* Words;
  Words from = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(from));
  constexpr int kWords = sizeof(LinearArgs) / 8;
  static_assert(sizeof(LinearArgs) % 8 == 0, "whole words");
  uint64_t words[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) words[i] = from[i];
  LinearArgs a;
  __builtin_memcpy(&a, words, sizeof(a));
  return a;
}

// Reads of steps' rows to LDS, one after the other.
template <class C>
struct StageLoader {
  static constexpr int kLoadRows = 8 * C::kWaves, kLoadsX = C::kX / kLoadRows, kLoadsW = C::kW / kLoadRows;
  const char *xb, *wb, *ab;
  int range_x, range_w, range_a;   // bytes from the wave's first row to the first byte of the last one
  int left;                        // bytes of a row from here to the part's end
  int64_t values;                  // bytes from the gates' rows to the values'
  int chunk16;
  uint32_t at[kLoadsX + kLoadsW], ahead;

  __device__ __forceinline__ void init(const TileAt& tile, int wave) {
    const LinearArgs p = args_anew();
    const int lane = lane_anew();
    const int k_begin = tile.part * p.part_bytes;
    const int k_end = p.row_bytes - k_begin < p.part_bytes ? p.row_bytes : k_begin + p.part_bytes;
    const int64_t m0 = (int64_t)tile.x * C::kX;
    const int n0 = tile.w * C::kOut;
    const int rows_x = p.n_rows - m0 < C::kX ? (int)(p.n_rows - m0) : C::kX;
    const int rows_w = p.n_out - n0 < C::kOut ? p.n_out - n0 : C::kOut;
    xb = p.x + m0 * p.x_row + k_begin;
    wb = p.w + (int64_t)n0 * p.w_row + k_begin;
    const char* vb = wb + (C::kGated ? (int64_t)p.n_out * p.w_row : 0);
    range_x = (int)((rows_x - 1) * p.x_row), range_w = (int)((rows_w - 1) * p.w_row);
    left = k_end - k_begin;
    // what this block asks for ahead
    const bool of_w = wave >= C::kWaves / 2;
    const int w4 = wave % (C::kWaves / 2);
    constexpr int kHalf = C::kWaves / 2, kRowsX = C::kX / kAheadW / kHalf, kRowsW = C::kW / kAheadX / kHalf;
    if (!of_w) {
      ab = xb, range_a = range_x;
      ahead = lane < kRowsX ? (uint32_t)((tile.w % kAheadW * kHalf + w4) * kRowsX + lane) * (uint32_t)p.x_row : kNowhere;
    } else {
      const bool value = C::kGated && w4 >= kHalf / 2;
      ab = value ? vb : wb, range_a = range_w;
      const int row = C::kGated ? (tile.x % kAheadX * (kHalf / 2) + w4 % (kHalf / 2)) * kRowsW + lane : (tile.x % kAheadX * kHalf + w4) * kRowsW + lane;
      ahead = lane < kRowsW ? (uint32_t)row * (uint32_t)p.w_row : kNowhere;
    }
    // Load i takes the rows 8 (wave + i kWaves) + lane / 8, its places lane % 8.  Of the weights' places every other 32
    // are values': with eight waves a wave's loads are all of gates' rows or all of values', 32 apart, with four they
    // alternate.
    static_assert(!C::kGated || C::kWaves == 8 || C::kWaves == 4, "gates or values");
    values = C::kGated ? (int64_t)p.n_out * p.w_row : 0;
    if (C::kGated && C::kWaves == 8 && ((wave >> 2) & 1)) wb = vb;
    chunk16 = ((lane ^ (lane >> 4) ^ (wave << 2)) & 7) * 16;
#pragma unroll
    for (int i = 0; i < kLoadsX; ++i) at[i] = (uint32_t)(i * kLoadRows + 8 * wave + (lane >> 3)) * (uint32_t)p.x_row + chunk16;
#pragma unroll
    for (int i = 0; i < kLoadsW; ++i)
      at[kLoadsX + i] = (uint32_t)((!C::kGated ? i * kLoadRows + 8 * wave : C::kWaves == 8 ? i * 32 + 8 * (wave & 3) : i / 2 * 32 + 8 * wave) + (lane >> 3)) * (uint32_t)p.w_row + chunk16;
  }
  // A step's loads.  Past the end nothing is read, and the places get zeros.
  __device__ __forceinline__ void load(char* lds, int wave) {
    const bool past = chunk16 >= left;
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)xb, 0, left > 0 ? range_x + left : 0, 0x00027000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)wb, 0, left > 0 ? range_w + left : 0, 0x00027000);
#pragma unroll
    for (int i = 0; i < kLoadsX; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (LdsVoid*)(lds + 8 * (wave + i * C::kWaves) * kStepBytes), 16, past ? kNowhere : at[i], 0, 0, 0);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(wb + values), 0, left > 0 ? range_w + left : 0, 0x00027000);
#pragma unroll
    for (int i = 0; i < kLoadsW; ++i) {
      LdsVoid* to = (LdsVoid*)(lds + (C::kX + 8 * (wave + i * C::kWaves)) * kStepBytes);
      const uint32_t from = past ? kNowhere : at[kLoadsX + i];
      if (C::kGated && C::kWaves == 4 && i % 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, to, 16, from, 0, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, to, 16, from, 0, 0, 0);
    }
    xb += kStepBytes, wb += kStepBytes, left -= kStepBytes;
  }
  // Asks for the lines of the step kAheadSteps after the one to be loaded next, so that they are in the L2 by then (`left` is that
  // one's).  Blocks that run at the same time on an XCD share rows: each asks for its part of them.  What arrives (4 bytes a
  // line) is of no use.
  __device__ __forceinline__ void ask(char* junk) {
    const int far = left - kAheadSteps * kStepBytes;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(ab + (C::kBuffers + kAheadSteps) * kStepBytes), 0, far > 0 ? range_a + far : 0, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid*)junk, 4, ahead, 0, 0, 0);
    ab += kStepBytes;
  }
};

// A wave's fragments of one part of a step.
template <class C>
struct Fragments {
  typename C::Op::Frag x[C::kBlocksX], w[C::kBlocksW];
  // lane_at: places of the lane's chunks in the first block's rows
  __device__ __forceinline__ void read(const char* xs, const char* ws, const int (&lane_at)[8 / C::kGroups], int part) {
    constexpr int kChunks = C::Op::kChunks, kBytes = C::Op::kBlock * kStepBytes;
#pragma unroll
    for (int i = 0; i < C::kFrags; ++i) {
      const char* from = i < C::kBlocksX ? xs + i * kBytes : ws + (i - C::kBlocksX) * kBytes;
      u32x4 c[kChunks];
#pragma unroll
      for (int q = 0; q < kChunks; ++q) c[q] = *reinterpret_cast<const u32x4*>(from + lane_at[part * kChunks + q]);
      if (i < C::kBlocksX) __builtin_memcpy(&x[i], c, sizeof(x[i]));
      else __builtin_memcpy(&w[i - C::kBlocksX], c, sizeof(w[0]));
    }
  }
};

// The order of a part's instructions: a read of LDS or a load from memory between any two products.  (8-bit products run
// four times as long as one is issued, and the compiler's own order is 2 % better.)
template <class C, int kDma>
__device__ __forceinline__ void beside_products() {
  if (C::Op::kChunks == 2) return;
  constexpr int kProducts = C::kBlocksX * C::kBlocksW * C::Op::kProducts;
  constexpr int kEach = kProducts / (2 * (C::kFrags + kDma)) > 1 ? kProducts / (2 * (C::kFrags + kDma)) : 1;
#pragma unroll
  for (int i = 0; i < C::kFrags; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, C::Op::kChunks, 0);
  }
#pragma unroll
  for (int i = 0; i < kDma; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);
  __builtin_amdgcn_sched_barrier(0);
}

template <class C>
__global__ __launch_bounds__(C::kThreads, C::kAtOnce * C::kWaves / 4) void k_linear_tiles(const LinearArgs args, int tiles_x, int tiles_w) {
  __shared__ __align__(16) char lds[C::kLds];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wx = wave / C::kWavesW, ww = wave % C::kWavesW;
  const int parts = args.parts;
  char* junk = lds + C::kBuffers * C::kStage + wave * 256;

  constexpr int kBlock = C::Op::kBlock;
  int lane_at[8 / C::kGroups];
#pragma unroll
  for (int s = 0; s < 8 / C::kGroups; ++s)
    lane_at[s] = lane % kBlock * kStepBytes + (((C::kGroups * s + lane / kBlock) ^ (lane % kBlock >> 1)) & 7) * 16;
  const int x_at = wx * C::kWaveX * kStepBytes, w_at = (C::kX + ww * C::kWaveW) * kStepBytes;

  const TileAt tile = tile_at(blockIdx.x, tiles_x, tiles_w, parts);
  StageLoader<C> in;
  in.init(tile, wave);
  const int steps = (in.left + kStepBytes - 1) / kStepBytes;
#pragma unroll
  for (int s = 0; s < C::kBuffers; ++s) in.load(lds + s * C::kStage, wave);
  typedef typename C::Op::Acc Acc;
  constexpr int kElements = 4 * C::Op::kQuads;
  Acc acc[C::kBlocksX][C::kBlocksW];
#pragma unroll
  for (int i = 0; i < C::kBlocksX; ++i)
#pragma unroll
    for (int j = 0; j < C::kBlocksW; ++j)
#pragma unroll
      for (int e = 0; e < kElements; ++e) acc[i][j][e] = 0.f;
  // float32: the sum of kTotalSteps steps is added to a total, so that roundings do not pile up over a long row
  Acc total[C::kTotals ? C::kBlocksX : 1][C::kTotals ? C::kBlocksW : 1];
  const auto add_to_total = [&] {
#pragma unroll
    for (int i = 0; i < (C::kTotals ? C::kBlocksX : 0); ++i)
#pragma unroll
      for (int j = 0; j < C::kBlocksW; ++j)
#pragma unroll
        for (int e = 0; e < kElements; ++e) total[i][j][e] += acc[i][j][e], acc[i][j][e] = 0.f;
  };
  if (C::kTotals) {
#pragma unroll
    for (int i = 0; i < C::kBlocksX; ++i)
#pragma unroll
      for (int j = 0; j < C::kBlocksW; ++j)
#pragma unroll
        for (int e = 0; e < kElements; ++e) total[C::kTotals ? i : 0][C::kTotals ? j : 0][e] = 0.f;
  }

  wait_all_but<(C::kBuffers - 1) * C::kLoads>();
  block_barrier();
  Fragments<C> f[2];
  char *now = lds, *next = lds + C::kStage;
  f[0].read(now + x_at, now + w_at, lane_at, 0);
  for (int k = 0; k < steps; ++k) {
#pragma unroll
    for (int s = 0; s < C::kParts; ++s) {
      if (s + 1 < C::kParts) {
        f[(s + 1) & 1].read(now + x_at, now + w_at, lane_at, s + 1);
        if (s == 0) in.ask(junk);
      } else {
        // every wave has read this step whole, and the next one has arrived: at most the loads of the steps after that and
        // what was asked for in this one are on their way
        wait_all_but<(C::kBuffers - 2) * C::kLoads + 1>();
        block_barrier();
        f[(s + 1) & 1].read(next + x_at, next + w_at, lane_at, 0);
        in.load(now, wave);
      }
#pragma unroll
      for (int e = 0; e < C::Op::kProducts; ++e)   // (the next product is on another sum)
#pragma unroll
        for (int i = 0; i < C::kBlocksX; ++i)
#pragma unroll
          for (int j = 0; j < C::kBlocksW; ++j) acc[i][j] = C::Op::mma(f[s & 1].w[j], f[s & 1].x[i], acc[i][j], e);
      if (s == 0) beside_products<C, 1>();
      else if (s + 1 < C::kParts) beside_products<C, 0>();
      else beside_products<C, C::kLoads>();
    }
    asm volatile("" ::: "memory");   // the next step's first fragments are read here, not where they are used
    now = next;
    next = next == lds + (C::kBuffers - 1) * C::kStage ? lds : next + C::kStage;
    if (C::kTotals && k % kTotalSteps == kTotalSteps - 1) add_to_total();
  }
  if (C::kTotals) {
    add_to_total();
#pragma unroll
    for (int i = 0; i < C::kBlocksX; ++i)
#pragma unroll
      for (int j = 0; j < C::kBlocksW; ++j) acc[i][j] = total[C::kTotals ? i : 0][C::kTotals ? j : 0];
  }
  wait_all_but<0>();   // the loads past the end write to LDS as well
  block_barrier();

  float* mine = reinterpret_cast<float*>(lds) + wave * C::kWaveFloats;
  // Through LDS, so that few lanes hold whole lines of the output: eight consecutive columns a lane.  16-byte chunk c of row
  // r lies at place c ^ r % 16 (c ^ r / 2 % 8 of rows of 8 chunks).
  const LinearArgs p = args_anew();
  const int64_t m0 = (int64_t)tile.x * C::kX + wx * C::kWaveX;
  constexpr int kCols = C::kOut / C::kWavesW, kLanes = kCols / 8, kRowsOnce = 64 / kLanes, kTimes = C::kPassRows < 2 * kRowsOnce ? 1 : 2;
  constexpr int kOneRows = 64 / kCols, kOneTimes = 4;
  static_assert(64 % kLanes == 0 && kCols <= 64 && C::kPassRows % (kTimes * kRowsOnce) == 0 && C::kPassRows % (kOneTimes * kOneRows) == 0, "whole rows");
  const int n0 = tile.w * C::kOut + ww * kCols;
  const auto place = [](int r, int c) { return r * C::kWaveW + (C::kWaveW == 64 ? c ^ (r & 15) : c ^ ((r >> 1) & 7)) * 4; };
  const int el = lane_anew(), col = el % kLanes * 8, row = el / kLanes, one = el % kCols;
  const bool whole = p.parts > 1 || (p.whole && n0 + kCols <= p.n_out);
  const auto row_in = [&](int64_t m) { return m < p.n_rows ? m : p.n_rows - 1; };
  Columns c;
  Column c1;
  if (whole && p.parts == 1) c.init<C::kGated>(p, n0 + col);
  if (!whole) c1.init<C::kGated>(p, n0 + one < p.n_out ? n0 + one : p.n_out - 1);
#pragma unroll
  for (int pass = 0; pass < C::kPasses; ++pass) {
    constexpr int kPassBlocks = C::kBlocksX / C::kPasses;
#pragma unroll
    for (int i = 0; i < kPassBlocks; ++i)
#pragma unroll
      for (int j = 0; j < C::kBlocksW; ++j)
#pragma unroll
        for (int q = 0; q < C::Op::kQuads; ++q) {
          const Acc& c4 = acc[pass * kPassBlocks + i][j];
          const f32x4 v = {c4[4 * q], c4[4 * q + 1], c4[4 * q + 2], c4[4 * q + 3]};
          *reinterpret_cast<f32x4*>(mine + place(i * kBlock + el % kBlock, (j * kBlock + q * C::Op::kStride) / 4 + el / kBlock)) = v;
        }
    __builtin_amdgcn_wave_barrier();   // (a wave's own LDS accesses are in order)
    const int64_t m1 = m0 + pass * C::kPassRows;
    if (whole) {
      RowAhead ahead[kTimes];
#pragma unroll
      for (int t = 0; t < kTimes; ++t)
        if (p.parts == 1) ahead[t].load(p, row_in(m1 + t * kRowsOnce + row), c.n);
#pragma unroll 1
      for (int r = row; r < C::kPassRows; r += kTimes * kRowsOnce) {
        RowAhead now_row[kTimes];
#pragma unroll
        for (int t = 0; t < kTimes; ++t) {
          now_row[t] = ahead[t];
          if (p.parts == 1) ahead[t].load(p, row_in(m1 + r + (kTimes + t) * kRowsOnce), c.n);   // (past the last one: not used)
        }
#pragma unroll
        for (int t = 0; t < kTimes; ++t) {
          const int at = r + t * kRowsOnce, from = C::kGated ? col / 32 * 64 + col % 32 : col;
          const int64_t m = m1 + at;
          float a[8], b[8];
          load_heads<4>(mine + place(at, from / 4), reinterpret_cast<float(&)[4]>(a[0]));
          load_heads<4>(mine + place(at, from / 4 + 1), reinterpret_cast<float(&)[4]>(a[4]));
          if (C::kGated) {
            load_heads<4>(mine + place(at, from / 4 + 8), reinterpret_cast<float(&)[4]>(b[0]));
            load_heads<4>(mine + place(at, from / 4 + 9), reinterpret_cast<float(&)[4]>(b[4]));
          }
          if (m >= p.n_rows) continue;
          if (p.parts > 1) {
            if (n0 + col < p.partial_cols) {
              float* o = p.partial + tile.part * p.partial_part + m * p.partial_cols * (C::kGated ? 2 : 1) + n0 + col;
              store_heads<8>(o, a);
              if (C::kGated) store_heads<8>(o + p.partial_cols, b);
            }
          } else {
            finish<C::kGated, C::kOnce>(p, c, m, now_row[t], a, b);
          }
        }
      }
    } else {
      const int from = C::kGated ? one / 32 * 64 + one % 32 : one;
#pragma unroll 1
      for (int r0 = el / kCols; r0 < C::kPassRows; r0 += kOneRows * kOneTimes) {
        OneAhead some[kOneTimes];
#pragma unroll
        for (int u = 0; u < kOneTimes; ++u) some[u].load(p, row_in(m1 + r0 + u * kOneRows), c1.n);
#pragma unroll
        for (int u = 0; u < kOneTimes; ++u) {
          const int r = r0 + u * kOneRows;
          const float a = mine[place(r, from / 4) + from % 4], b = C::kGated ? mine[place(r, from / 4 + 8) + from % 4] : 0.f;
          if (m1 + r < p.n_rows && n0 + one < p.n_out) finish_one<C::kGated>(p, c1, m1 + r, some[u], a, b);
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace gc
