// The attention kernels: waves that share a tile of keys and have rows of
// their own, and waves that share the rows and have keys of their own.
#pragma once

#include <type_traits>

#include "gc_attention_core.h"

namespace gc {

// Until the wave's reads of LDS have arrived.
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
  asm volatile("" ::: "memory");
}

// A barrier that waits for no memory operation itself (__syncthreads waits
// for all loads to LDS, the next tiles' among them).
__device__ __forceinline__ void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Four channels of a finished row.
__device__ __forceinline__ void store4(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }
__device__ __forceinline__ void store4(uint16_t* p, f32x4 x) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
}

// One row's result from its weighted sum (by four channels), maximum and sum.
struct Normaliser {
  float inv, lse;
  __device__ __forceinline__ Normaliser(float m, float l) {
    // l is 0 for a row without a key, or with scores of -inf alone
    inv = l == 0.f ? 0.f : 1.f / l;
    lse = l == 0.f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
};

// Results of a wave's rows (l whole, not a lane's part): to the output, or as
// a part of rows whose keys are split.
template <class T, int kDim, class C>
__device__ __forceinline__ void store_rows(const AttentionArgs& p, const AttentionItem& it, int kv_head, const C& core,
                                           float l, int first_row, int tile_rows, int lane) {
  const int half = lane >> 5;
  const int local = first_row + (lane & 31);
  if (it.parts > 1) {
    float* part = p.partial + ((int64_t)it.slot * p.kv_heads + kv_head) * ((int64_t)tile_rows * (kDim + 2));
    float* row = part + (int64_t)local * kDim;
#pragma unroll
    for (int d = 0; d < C::kOut; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4(row + 32 * d + 8 * g + 4 * half,
               f32x4{core.o[d][4 * g], core.o[d][4 * g + 1], core.o[d][4 * g + 2], core.o[d][4 * g + 3]});
    if (half == 0) *reinterpret_cast<float2*>(part + (int64_t)tile_rows * kDim + 2 * local) = float2{core.m, l};
    return;
  }
  const RowOf r = row_of(p, it, kv_head, it.row0 + local);
  if (!r.live) return;
  const Normaliser z(core.m, l);
  T* row = (T*)p.out + r.token * p.o_token + (int64_t)r.head * p.o_head;
#pragma unroll
  for (int d = 0; d < C::kOut; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * d + 8 * g + 4 * half;
      if (c < p.dim) {
        f32x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : core.o[d][4 * g + j] * z.inv;
        store4(row + c, x);
      }
    }
  if (p.lse && half == 0) p.lse[(int64_t)r.head * p.total_q + r.token] = z.lse;
}

// Adds the parts of split rows, in their order: a launch of its own after the
// parts', one block for kJoin runs of four channels of one tile (blocks of
// items that are not their tile's first part have nothing to do).  (Joined by the last of a
// tile's blocks instead, 2048 tokens x 16 heads x 64 in two parts took 48 us, 160 rows over 9000 keys in 18
// parts 74 us: that block alone waits for one load after the other.)
constexpr int kJoin = 256;

template <class T, int kDim>
__global__ __launch_bounds__(kJoin) void k_attention_join(const AttentionArgs p, int tile_rows) {
  const int kv_head = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];
  if (it.parts < 2 || it.slot != it.slot0) return;
  const int rows = it.rows - it.row0 < tile_rows ? it.rows - it.row0 : tile_rows;
  const int e = blockIdx.y * kJoin + threadIdx.x, local = e / (kDim / 4), c = e % (kDim / 4) * 4;
  if (local >= rows || c >= p.dim) return;
  const int64_t stride = (int64_t)tile_rows * (kDim + 2) * p.kv_heads;   // from part to part
  const float* first = p.partial + ((int64_t)it.slot0 * p.kv_heads + kv_head) * ((int64_t)tile_rows * (kDim + 2));
  const float* ml = first + (int64_t)tile_rows * kDim + 2 * local;
  const float* row = first + (int64_t)local * kDim + c;
  // with the maxima as they come, four parts' loads together
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < it.parts; i0 += 4) {
    float2 x[4];
    f32x4 y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = (i0 + i < it.parts ? i0 + i : i0) * stride;
      x[i] = *reinterpret_cast<const float2*>(ml + at);
      y[i] = *reinterpret_cast<const f32x4*>(row + at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i0 + i >= it.parts) continue;
      const float mn = fmaxf(m, x[i].x), ms = mn == -__builtin_inff() ? 0.f : mn;
      const float f = sum_factor(m - ms), g = sum_factor(x[i].x - ms);
      m = mn;
      l = l * f + x[i].y * g;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * f + y[i][j] * g;
    }
  }
  const RowOf r = row_of(p, it, kv_head, it.row0 + local);
  const Normaliser z(m, l);
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : o[j] * z.inv;
  store4((T*)p.out + r.token * p.o_token + (int64_t)r.head * p.o_head + c, o);
  if (p.lse && c == 0) p.lse[(int64_t)r.head * p.total_q + r.token] = z.lse;
}

template <class T, int kDim>
void launch_join(const AttentionArgs& p, int tile_rows, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL((k_attention_join<T, kDim>), dim3(blocks, (unsigned)(tile_rows * (kDim / 4) / kJoin)), dim3(kJoin), 0, stream, p,
                     tile_rows);
}

// ---------------------------------------------------------------------------
// rows, bfloat16: the waves of a block hold 32 rows each and walk the same
// keys.  A wave's work at tile i has two parts, each of matrix products beside
// vector work that does not need them: tile i - 1's values with tile i's
// maximum, then tile i + 1's scores with tile i's weights
// (values_and_maximum, weights_and_scores).  K tiles lie in two places in
// turn, V tiles in four.
//
// At tile i the block has passed a barrier after which K of i + 1 and V of i
// are there, and nobody reads K of i or V of i - 2 any more: K of i + 2 and V
// of i + 2 are asked for in their places.  The next barrier waits for that K
// and for the V asked for a tile before; the last V may be outstanding.
//
// What bounds it: with 64 channels the issue of both kinds (while a compute
// unit has work its vector units are busy 67 % of the time, its matrix units 41 %; a lone wave takes 34
// cycles for a product, 46 for four multiply-adds, two exponentials and a
// conversion, and 54 for all) and the launch's incomplete last round (688 blocks for 256 compute units that hold one
// each: 2.7 rounds take 3), with 128 the power that the products draw (busy 56 % and 67 %, the
// clock at 1.8 of 2.4 GHz; the products alone take 2.9 of the 4.1 ms).
// 64 keys a tile up to 128 channels, 32 above (and with four waves a block
// above 96): what registers and LDS hold.  24576 tokens x 16 heads x 128: 4.1
// ms, 1220 TFLOP/s; 10403 tokens in four sequences x 16 x 64: 145 us (boxes differ by up to 7 %).  Not faster (against 4.27 ms and 707 us at the time):
// halves of the block that take turns at products and vector work, with a
// barrier a part (4.36 ms, causal 810 us); 32 keys a tile at three waves a SIMD for 64 channels
// (1213 us against 1154); weights against a maximum that only the sum checks
// (4.7 ms); wave priorities, operands 2, 6 or 8 products ahead (within 1 %).
// ---------------------------------------------------------------------------
template <int kDim, int kKeyBlocks, int kWaves>
__device__ __forceinline__ void attention_rows(const AttentionArgs& p) {
  using T = uint16_t;
  constexpr int kKeys = 32 * kKeyBlocks, kTile = kKeys * kDim * (int)sizeof(T), kRows = 32 * kWaves;
  // an array a tile: the compiler then sees that a read of one does not wait for the loads to another
  __shared__ __attribute__((aligned(1024))) char k0[kTile], k1[kTile], v0[kTile], v1[kTile], v2[kTile], v3[kTile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_head = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];

  using C = Core<T, kDim, kKeyBlocks>;
  C core;
  core.init();
  core.init_values(lane);
  const int first_row = wave * 32;
  const RowOf r = row_of(p, it, kv_head, it.row0 + first_row + (lane & 31));
  const int limit = r.limit < it.k_end ? r.limit : it.k_end;
  core.load_q((const T*)p.q + r.token * p.q_token + (int64_t)r.head * p.q_head, p.dim, lane >> 5);

  using Loader = TileLoader<T, kDim, kKeys, kWaves>;
  Loader kl, vl;
  // (to the sequence's end, not the part's: what a part's last tile holds past it is masked)
  kl.init(p.k, it.k_token0, p.k_token, kv_head * p.k_head, p.dim, it.k_begin, it.k_len, wave, lane);
  vl.init(p.v, it.k_token0, p.v_token, kv_head * p.v_head, p.dim, it.k_begin, it.k_len, wave, lane);
  // the wave's rows see at most high keys, the block's rows at least low (limits grow with the row)
  const int high = __builtin_amdgcn_readlane(limit, 31);
  int low = it.k_end;
  if (p.causal) {
    const int least = it.row0 / p.group + it.reach;
    low = least < low ? least : low;
  }
  const float c = p.scale * kLog2e;

  int key0 = it.k_begin;
  typename C::S even, odd;   // scores of even and odd tiles
  typename C::Weights w;
  typename C::Operands x;
  float mx, ms;
  uint32_t bad = 0;
  int first_masked = key0;

  if (key0 < it.k_end) {
    kl.load(k0, wave);
    kl.load(k1, wave);
    vl.load(v0, wave);
    vl.load(v1, wave);
    wait_loads<0>();
    __syncthreads();
    core.scores(k0, lane, even);
    __syncthreads();
    kl.load(k0, wave);
    vl.load(v2, wave);
    mask(even, key0, limit, lane);
    maximum(even, mx);
    update_maximum(core, mx, c, ms);
    core.weights(even, c, ms, w);
    core.scores(k1, lane, odd);
    wait_lds();   // (a product, and its operand's wait, may be moved past a barrier that waits for nothing)
    key0 += kKeys;
  }
  const auto arrive = [&] {
    wait_loads<Loader::kMine>();
    barrier_only();
  };
  // tile i at key0, nothing masked in it nor before it
  const auto tile = [&](typename C::S& now, typename C::S& next, char* k_now, char* k_next, char* v_before, char* v_now, char* v_after) {
    arrive();
    kl.load(k_now, wave);
    vl.load(v_after, wave);
    core.values_and_maximum(x, v_before, w, now, k_next, lane, mx);
    update_maximum(core, mx, c, ms);
    core.weights_and_scores(x, now, c, ms, w, k_next, next, v_now, lane);
    key0 += kKeys;
  };
  int phase = 1;   // i % 4
  if (key0 + kKeys <= low) {
    core.first_values(v0, x);
    while (key0 + 4 * kKeys <= low) {
      tile(odd, even, k1, k0, v0, v1, v3);
      tile(even, odd, k0, k1, v1, v2, v0);
      tile(odd, even, k1, k0, v2, v3, v1);
      tile(even, odd, k0, k1, v3, v0, v2);
    }
    // up to three more
    if (key0 + kKeys <= low) {
      tile(odd, even, k1, k0, v0, v1, v3);
      phase = 2;
      if (key0 + kKeys <= low) {
        tile(even, odd, k0, k1, v1, v2, v0);
        phase = 3;
        if (key0 + kKeys <= low) {
          tile(odd, even, k1, k0, v2, v3, v1);
          phase = 0;
        }
      }
    }
  }
  // the other tiles: scores are masked, and values that are not finite left out
  if (it.k_begin < it.k_end) {
    first_masked = key0 - kKeys;
    if (phase & 1) even = odd;
    while (key0 < it.k_end) {
      wait_lds();   // as above, for this loop's reads
      arrive();
      char* const k_now = phase & 1 ? k1 : k0;
      kl.load(k_now, wave);
      vl.load(phase == 0 ? v2 : phase == 1 ? v3 : phase == 2 ? v0 : v1, wave);
      if (key0 - kKeys < high) bad |= core.add_masked(phase == 0 ? v3 : phase == 1 ? v0 : phase == 2 ? v1 : v2, lane, w);
      if (key0 < high) {
        mask(even, key0, limit, lane);
        maximum(even, mx);
        update_maximum(core, mx, c, ms);
        core.weights(even, c, ms, w);
        core.scores(phase & 1 ? k0 : k1, lane, even);
      }
      key0 += kKeys;
      phase = (phase + 1) & 3;
    }
    wait_loads<0>();
    __syncthreads();
    if (key0 - kKeys < high) bad |= core.add_masked(phase == 0 ? v3 : phase == 1 ? v0 : phase == 2 ? v1 : v2, lane, w);
  }

  const float l = sum_halves(core.l);
  if (__any(bad != 0)) add_nonfinite<T>(p, it, kv_head, core, first_masked, high, kKeys, kKeys, limit, lane);
  settle_nonfinite<T>(p, it, kv_head, core, l, it.k_begin, high, 64, 64, limit, lane);
  store_rows<T, kDim>(p, it, kv_head, core, l, first_row, kRows, lane);
}

template <int kDim, int kKeyBlocks, int kWaves, int kPerSimd>
__global__ __launch_bounds__(64 * kWaves, kPerSimd) void k_attention_rows(const AttentionArgs p) {
  attention_rows<kDim, kKeyBlocks, kWaves>(p);
}

// ---------------------------------------------------------------------------
// rows, float32: a product takes sixteen times as long as bfloat16's, so a
// tile's parts follow one another and the blocks of a compute unit (or its
// four waves) fill the gaps.  Two places for K and V each: one tile is worked
// on while the next arrives.  1024 + 1 + 517 + 770 tokens x 8 heads x 64: 51
// us, of which the parts' join takes 7.  There two blocks share a compute unit
// (512 for 256), and while one has work its matrix units are busy 74 % of the time: two waves
// a SIMD do not fill the gaps between scores, weights and values, and each tile has a barrier.
// Slower: the next tile's scores beside this tile's weights (60 us; 2000
// tokens x 8 x 256 404 against 289): the compiler then waits for the loads to
// LDS inside a tile.
// ---------------------------------------------------------------------------
template <int kDim, int kPerSimd>
__global__ __launch_bounds__(256, kPerSimd) void k_attention_rows_f32(const AttentionArgs p) {
  constexpr int kWaves = 4, kKeys = 32, kTile = kKeys * kDim * 4, kRows = 32 * kWaves;
  __shared__ __attribute__((aligned(1024))) char k0[kTile], k1[kTile], v0[kTile], v1[kTile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_head = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];

  using C = Core<float, kDim, 1>;
  C core;
  core.init();
  core.init_values(lane);
  const int first_row = wave * 32;
  const RowOf r = row_of(p, it, kv_head, it.row0 + first_row + (lane & 31));
  const int limit = r.limit < it.k_end ? r.limit : it.k_end;
  core.load_q((const float*)p.q + r.token * p.q_token + (int64_t)r.head * p.q_head, p.dim, lane >> 5);

  TileLoader<float, kDim, kKeys, kWaves> kl, vl;
  kl.init(p.k, it.k_token0, p.k_token, kv_head * p.k_head, p.dim, it.k_begin, it.k_len, wave, lane);
  vl.init(p.v, it.k_token0, p.v_token, kv_head * p.v_head, p.dim, it.k_begin, it.k_len, wave, lane);
  const int high = __builtin_amdgcn_readlane(limit, 31);
  int low = it.k_end;
  if (p.causal) {
    const int least = it.row0 / p.group + it.reach;
    low = least < low ? least : low;
  }
  const float c = p.scale * kLog2e;

  int key0 = it.k_begin;
  uint32_t bad = 0;
  const auto tile = [&](auto masked, const char* k_now, const char* v_now, char* k_next, char* v_next) {
    constexpr bool kMasked = decltype(masked)::value;
    wait_loads<0>();
    __syncthreads();   // this tile is there, and nobody reads the other one
    kl.load(k_next, wave);
    vl.load(v_next, wave);
    if (!kMasked || key0 < high) {
      typename C::S s;
      typename C::Weights w;
      float mx, ms;
      core.scores(k_now, lane, s);
      if constexpr (kMasked) mask(s, key0, limit, lane);
      maximum(s, mx);
      update_maximum(core, mx, c, ms);
      core.weights(s, c, ms, w);
      if constexpr (kMasked) bad |= core.add_masked(v_now, lane, w);
      else core.add_values(v_now, lane, w);
    }
    key0 += kKeys;
  };
  if (key0 < it.k_end) {
    kl.load(k0, wave);
    vl.load(v0, wave);
  }
  while (key0 + 2 * kKeys <= low) {
    tile(std::false_type{}, k0, v0, k1, v1);
    tile(std::false_type{}, k1, v1, k0, v0);
  }
  const int first_masked = key0;
  for (bool other = false; key0 < it.k_end; other = !other) {
    if (other) tile(std::true_type{}, k1, v1, k0, v0);
    else tile(std::true_type{}, k0, v0, k1, v1);
  }
  wait_loads<0>();   // before the block's LDS is given up

  const float l = sum_halves(core.l);
  if (__any(bad != 0)) add_nonfinite<float>(p, it, kv_head, core, first_masked, high, kKeys, kKeys, limit, lane);
  settle_nonfinite<float>(p, it, kv_head, core, l, it.k_begin, high, 64, 64, limit, lane);
  store_rows<float, kDim>(p, it, kv_head, core, l, first_row, kRows, lane);
}

// ---------------------------------------------------------------------------
// keys: few rows over many keys.  The waves of a block hold the same 32 rows
// and take tiles of 32 keys in turn, each with two tiles of its own in LDS
// and no barrier until the end, where their results are added.  Bound by the
// read of the keys and values: 495 MB for 8 tokens (32 heads on 8 of 128) in
// 84 us, 5.9 TB/s where a large read reaches 7.0, and 5 us for the join.  Not
// so in float32 above 64 channels, where two waves or one a compute unit are bound by their products on 32 rows:
// 16 tokens (32 heads on 8) over 4096 keys each take 54, 144, 379 and 1065 us
// at 64, 128, 192 and 256 channels (the last spills), where the reads take 38, 77, 115 and 153.
// ---------------------------------------------------------------------------
template <class T, int kDim, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kDim * sizeof(T) <= 64 ? 4 : 1) void k_attention_keys(const AttentionArgs p) {
  constexpr int kKeys = 32, kTile = kKeys * kDim * (int)sizeof(T);
  // the loads that may be outstanding where a tile is needed: the three asked for after it (the counter's
  // range is 63: where they are more, a few of them are waited for too)
  constexpr int kLoads = TileLoader<T, kDim, kKeys, 1>::kMine, kLeft = 3 * kLoads < 63 ? 3 * kLoads : 63;
  static_assert(32 * kDim * 4 <= 4 * kTile, "a wave's result fits its tiles");
  __shared__ __attribute__((aligned(1024))) char lds[kWaves * 4 * kTile];
  __shared__ float ml[kWaves][32][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_head = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];
  char* mine = lds + wave * 4 * kTile;

  // Tile i of the wave: K at mine + i % 2 * 2 kTile, V behind it.  Two tiles
  // are on their way at any time: a K tile's successor but one is asked for as soon
  // as its scores are in registers, a V tile's as soon as its products are issued.
  TileLoader<T, kDim, kKeys, 1, kWaves, true> kl, vl;
  const int first = it.k_begin + wave * kKeys;
  constexpr int kStep = kWaves * kKeys;
  kl.init(p.k, it.k_token0, p.k_token, kv_head * p.k_head, p.dim, first, it.k_len, 0, lane);
  vl.init(p.v, it.k_token0, p.v_token, kv_head * p.v_head, p.dim, first, it.k_len, 0, lane);
  using C = Core<T, kDim, 1>;
  C core;
  core.init();
  core.init_values(lane);
  const RowOf r = row_of(p, it, kv_head, it.row0 + (lane & 31));
  const int limit = r.limit < it.k_end ? r.limit : it.k_end;
  core.load_q((const T*)p.q + r.token * p.q_token + (int64_t)r.head * p.q_head, p.dim, lane >> 5);
  if (first < it.k_end) {
    kl.load(mine, 0);
    vl.load(mine + kTile, 0);
    kl.load(mine + 2 * kTile, 0);
    vl.load(mine + 3 * kTile, 0);
  }
  const int low = __builtin_amdgcn_readfirstlane(limit);
  const int high = __builtin_amdgcn_readlane(limit, 31);
  const float c = p.scale * kLog2e;

  int stage = 0;
  const auto tile = [&](int key0, auto masked) {
    constexpr bool kMasked = decltype(masked)::value;
    char* kt = mine + stage * 2 * kTile;
    typename C::S s;
    typename C::Weights w;
    float mx, ms;
    wait_loads<kLeft>();
    core.scores(kt, lane, s);
    wait_lds();
    kl.load(kt, 0);
    if constexpr (kMasked) mask(s, key0, limit, lane);
    maximum(s, mx);
    update_maximum(core, mx, c, ms);
    core.weights(s, c, ms, w);
    wait_loads<kLeft>();
    uint32_t left_out = 0;
    if constexpr (kMasked) left_out = core.add_masked(kt + kTile, lane, w);
    else core.add_values(kt + kTile, lane, w);
    wait_lds();
    vl.load(kt + kTile, 0);
    stage ^= 1;
    return left_out;
  };
  int key0 = first;
  for (; key0 + kKeys <= low; key0 += kStep) tile(key0, std::false_type{});
  const int first_masked = key0;
  uint32_t bad = 0;
  for (; key0 < high; key0 += kStep) bad |= tile(key0, std::true_type{});
  if (__any(bad != 0))
    add_nonfinite<T>(p, it, kv_head, core, first_masked, high, kKeys, kWaves * kKeys, limit, lane);
  float l = sum_halves(core.l);
  settle_nonfinite<T>(p, it, kv_head, core, l, first, high, kKeys, kStep, limit, lane);
  // the waves' results, added by the first wave in their order
  wait_loads<0>();   // (also before the block's LDS is given up)
  if constexpr (kWaves > 1) {
    float* o = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[(d * 16 + i) * 64 + lane] = core.o[d][i];
    if (lane < 32) {
      ml[wave][lane][0] = core.m;
      ml[wave][lane][1] = l;
    }
    __syncthreads();
    if (wave == 0) {
      float m = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][lane & 31][0]);
      const float ms = m == -__builtin_inff() ? 0.f : m;
      l = 0.f;
#pragma unroll
      for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) core.o[d][i] = 0.f;
      for (int w = 0; w < kWaves; ++w) {
        const float f = sum_factor(ml[w][lane & 31][0] - ms);
        l += ml[w][lane & 31][1] * f;
        const float* x = reinterpret_cast<const float*>(lds + w * 4 * kTile);
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) core.o[d][i] += x[(d * 16 + i) * 64 + lane] * f;
      }
      core.m = m;
    }
  }
  if (wave == 0) store_rows<T, kDim>(p, it, kv_head, core, l, 0, 32, lane);
}

}  // namespace gc
