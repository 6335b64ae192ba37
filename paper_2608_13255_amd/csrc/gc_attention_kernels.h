// The attention kernels: waves that share a tile of keys and have rows of
// their own, and waves that share the rows and have keys of their own.
#pragma once

#include <type_traits>

#include "gc_attention_core.h"

namespace gc {

// Until at most kLeft of the wave's loads are outstanding.
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  static_assert(kLeft < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | (7 << 4) | (15 << 8) | ((kLeft >> 4) << 14));
  asm volatile("" ::: "memory");
}

// Until the wave's reads of LDS have arrived.
__device__ __forceinline__ void wait_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
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
template <class T, int kDim, class C, int kNq>
__device__ __forceinline__ void store_rows(const AttentionArgs& p, const AttentionItem& it, int kv_head, const C& core,
                                           const float (&l)[kNq], int first_row, int tile_rows, int lane) {
  const int half = lane >> 5;
#pragma unroll
  for (int n = 0; n < kNq; ++n) {
    const int local = first_row + n * 32 + (lane & 31);
    if (it.parts > 1) {
      float* part = p.partial + ((int64_t)it.slot * p.kv_heads + kv_head) * ((int64_t)tile_rows * (kDim + 2));
      float* row = part + (int64_t)local * kDim;
#pragma unroll
      for (int d = 0; d < C::kOut; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          store4(row + 32 * d + 8 * g + 4 * half,
                 f32x4{core.o[n][d][4 * g], core.o[n][d][4 * g + 1], core.o[n][d][4 * g + 2], core.o[n][d][4 * g + 3]});
      if (half == 0) {
        float* ml = part + (int64_t)tile_rows * kDim + 2 * local;
        ml[0] = core.m[n];
        ml[1] = l[n];
      }
    } else {
      const RowOf r = row_of(p, it, kv_head, it.row0 + local);
      if (!r.live) continue;
      const Normaliser z(core.m[n], l[n]);
      T* row = (T*)p.out + r.token * p.o_token + (int64_t)r.head * p.o_head;
#pragma unroll
      for (int d = 0; d < C::kOut; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int c = 32 * d + 8 * g + 4 * half;
          if (c < p.dim) {
            f32x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = z.inv == 0.f && l[n] == 0.f ? 0.f : core.o[n][d][4 * g + j] * z.inv;
            store4(row + c, x);
          }
        }
      if (p.lse && half == 0) p.lse[(int64_t)r.head * p.total_q + r.token] = z.lse;
    }
  }
}

// After a block has written its part of split rows: the last of the tile's
// blocks to finish adds the parts, in their order, and leaves the counter at
// zero for the next call.  Every block's stores are complete and
// released before its count; the last one's reads come after it has acquired
// all of them.
template <class T, int kDim>
__device__ __forceinline__ void join_parts(const AttentionArgs& p, const AttentionItem& it, int kv_head, int tile_rows) {
  __shared__ uint32_t last;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
  __syncthreads();
  uint32_t* counter = p.counters + (int64_t)it.group_id * p.kv_heads + kv_head;
  if (threadIdx.x == 0)
    last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == (uint32_t)it.parts;
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int64_t stride = (int64_t)tile_rows * (kDim + 2);
  const float* first = p.partial + ((int64_t)it.slot0 * p.kv_heads + kv_head) * stride;
  const int rows = it.rows - it.row0 < tile_rows ? it.rows - it.row0 : tile_rows;
  for (int e = threadIdx.x; e < rows * (kDim / 4); e += blockDim.x) {
    const int local = e / (kDim / 4), c = (e % (kDim / 4)) * 4;
    if (c >= p.dim) continue;
    const float* ml = first + (int64_t)tile_rows * kDim + 2 * local;
    float m = -__builtin_inff();
    for (int i = 0; i < it.parts; ++i) m = fmaxf(m, ml[i * stride * p.kv_heads]);
    const float ms = m == -__builtin_inff() ? 0.f : m;
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < it.parts; ++i) {
      const int64_t at = i * stride * p.kv_heads;
      const float f = exp2_hw(ml[at] - ms);
      l += ml[at + 1] * f;
      const f32x4 x = *reinterpret_cast<const f32x4*>(first + at + (int64_t)local * kDim + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += x[j] * f;
    }
    const RowOf r = row_of(p, it, kv_head, it.row0 + local);
    const Normaliser z(m, l);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : o[j] * z.inv;
    store4((T*)p.out + r.token * p.o_token + (int64_t)r.head * p.o_head + c, o);
    if (p.lse && c == 0) p.lse[(int64_t)r.head * p.total_q + r.token] = z.lse;
  }
}

// The weights of one tile and their values.  Without kMasked every row of the
// wave sees all of the tile.  Returns whether values were left out
// (add_nonfinite).
template <bool kMasked, int kKeyBlocks, class C, int kNq>
__device__ __forceinline__ uint32_t tile_step(C& core, const char* kt, const char* vt, float c, int key0, const int (&limit)[kNq],
                                              int lane) {
  f32x16 s[kNq][kKeyBlocks];
  core.scores(kt, lane, s);
  softmax_tile<kMasked>(core, s, c, key0, limit, lane);
  return core.template add_values<kMasked>(vt, lane, s);
}

// ---------------------------------------------------------------------------
// rows: the waves of a block hold 32 kNq rows each and walk the same keys,
// two tiles in LDS: one is worked on while the next arrives.
// ---------------------------------------------------------------------------
template <class T, int kDim, int kNq, int kKeyBlocks, int kWaves, int kPerSimd>
__global__ __launch_bounds__(64 * kWaves, kPerSimd) void k_attention_rows(const AttentionArgs p) {
  constexpr int kKeys = 32 * kKeyBlocks, kTile = kKeys * kDim * (int)sizeof(T), kRows = 32 * kNq * kWaves;
  __shared__ __attribute__((aligned(1024))) char lds[4 * kTile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_head = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];

  TileLoader<T, kDim, kKeys, kWaves> kl, vl;
  kl.init(p.k, it.k_token0, p.k_token, kv_head * p.k_head, p.dim, wave, lane);
  vl.init(p.v, it.k_token0, p.v_token, kv_head * p.v_head, p.dim, wave, lane);

  Core<T, kDim, kNq, kKeyBlocks> core;
  core.init();
  const int first_row = wave * 32 * kNq;
  int limit[kNq];
#pragma unroll
  for (int n = 0; n < kNq; ++n) {
    const RowOf r = row_of(p, it, kv_head, it.row0 + first_row + n * 32 + (lane & 31));
    limit[n] = r.limit < it.k_end ? r.limit : it.k_end;
    core.load_q(n, (const T*)p.q + r.token * p.q_token + (int64_t)r.head * p.q_head, p.dim, lane >> 5);
  }
  if (it.k_begin < it.k_end) {
    kl.load(lds, it.k_begin, it.k_len, wave);
    vl.load(lds + kTile, it.k_begin, it.k_len, wave);
  }
  // the wave's rows see at most high keys, the block's rows at least low (limits grow with the row)
  const int high = __builtin_amdgcn_readlane(limit[kNq - 1], 31);
  int low = it.k_end;
  if (p.causal) {
    const int least = it.row0 / p.group + it.reach;
    low = least < low ? least : low;
  }
  const float c = p.scale * kLog2e;

  int stage = 0;
  // the tile at key0 is there and nobody reads the other one, which the next one goes to
  const auto next = [&](int key0) {
    wait_loads<0>();
    __syncthreads();
    char* kt = lds + stage * 2 * kTile;
    stage ^= 1;
    if (key0 + kKeys < it.k_end) {
      kl.load(lds + stage * 2 * kTile, key0 + kKeys, it.k_len, wave);
      vl.load(lds + stage * 2 * kTile + kTile, key0 + kKeys, it.k_len, wave);
    }
    return kt;
  };
  int key0 = it.k_begin;
  for (; key0 + kKeys <= low; key0 += kKeys) {
    const char* kt = next(key0);
    tile_step<false, kKeyBlocks>(core, kt, kt + kTile, c, key0, limit, lane);
  }
  const int first_masked = key0;
  uint32_t bad = 0;
  for (; key0 < it.k_end; key0 += kKeys) {
    const char* kt = next(key0);
    if (key0 < high) bad |= tile_step<true, kKeyBlocks>(core, kt, kt + kTile, c, key0, limit, lane);
  }

  if (__any(bad != 0)) {
    add_nonfinite<T>(core, vl.base, vl.stride, p.dim, first_masked, high, kKeys, kKeys, limit, lane);
  }
  float l[kNq];
#pragma unroll
  for (int n = 0; n < kNq; ++n) l[n] = sum_halves(core.l[n]);
  store_rows<T, kDim>(p, it, kv_head, core, l, first_row, kRows, lane);
  if (it.parts > 1) join_parts<T, kDim>(p, it, kv_head, kRows);
}

// ---------------------------------------------------------------------------
// keys: few rows over many keys.  The waves of a block hold the same 32 rows
// and take tiles of 32 keys in turn, each with two tiles of its own in LDS
// and no barrier until the end, where their results are added.
// ---------------------------------------------------------------------------
template <class T, int kDim, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void k_attention_keys(const AttentionArgs p) {
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
  TileLoader<T, kDim, kKeys, 1> kl, vl;
  kl.init(p.k, it.k_token0, p.k_token, kv_head * p.k_head, p.dim, 0, lane);
  vl.init(p.v, it.k_token0, p.v_token, kv_head * p.v_head, p.dim, 0, lane);
  const int first = it.k_begin + wave * kKeys;
  constexpr int kStep = kWaves * kKeys;
  const int last_key = it.k_len - 1;
  // past the wave's last tile the loads go on, from a tile that is there, so that the counts below hold
  const auto load_k = [&](int key0, int stage) { kl.load(mine + stage * 2 * kTile, key0 < it.k_end ? key0 : last_key, it.k_len, 0); };
  const auto load_v = [&](int key0, int stage) { vl.load(mine + stage * 2 * kTile + kTile, key0 < it.k_end ? key0 : last_key, it.k_len, 0); };
  Core<T, kDim, 1, 1> core;
  core.init();
  const RowOf r = row_of(p, it, kv_head, it.row0 + (lane & 31));
  const int limit[1] = {r.limit < it.k_end ? r.limit : it.k_end};
  core.load_q(0, (const T*)p.q + r.token * p.q_token + (int64_t)r.head * p.q_head, p.dim, lane >> 5);
  if (first < it.k_end) {
    load_k(first, 0);
    load_v(first, 0);
    load_k(first + kStep, 1);
    load_v(first + kStep, 1);
  }
  const int low = __builtin_amdgcn_readfirstlane(limit[0]);
  const int high = __builtin_amdgcn_readlane(limit[0], 31);
  const float c = p.scale * kLog2e;

  int stage = 0;
  const auto tile = [&](int key0, auto masked) {
    constexpr bool kMasked = decltype(masked)::value;
    char* kt = mine + stage * 2 * kTile;
    f32x16 s[1][1];
    wait_loads<kLeft>();
    core.scores(kt, lane, s);
    wait_lds();
    load_k(key0 + 2 * kStep, stage);
    softmax_tile<kMasked>(core, s, c, key0, limit, lane);
    wait_loads<kLeft>();
    const uint32_t left_out = core.template add_values<kMasked>(kt + kTile, lane, s);
    wait_lds();
    load_v(key0 + 2 * kStep, stage);
    stage ^= 1;
    return left_out;
  };
  int key0 = first;
  for (; key0 + kKeys <= low; key0 += kStep) tile(key0, std::false_type{});
  const int first_masked = key0;
  uint32_t bad = 0;
  for (; key0 < high; key0 += kStep) bad |= tile(key0, std::true_type{});
  if (__any(bad != 0))
    add_nonfinite<T>(core, vl.base, vl.stride, p.dim, first_masked, high, kKeys, kWaves * kKeys, limit, lane);
  // the waves' results, added by the first wave in their order
  float l[1] = {sum_halves(core.l[0])};
  wait_loads<0>();   // (also before the block's LDS is given up)
  if constexpr (kWaves > 1) {
    float* o = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[(d * 16 + i) * 64 + lane] = core.o[0][d][i];
    if (lane < 32) {
      ml[wave][lane][0] = core.m[0];
      ml[wave][lane][1] = l[0];
    }
    __syncthreads();
    if (wave == 0) {
      float m = -__builtin_inff();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][lane & 31][0]);
      const float ms = m == -__builtin_inff() ? 0.f : m;
      l[0] = 0.f;
#pragma unroll
      for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) core.o[0][d][i] = 0.f;
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_hw(ml[w][lane & 31][0] - ms);
        l[0] += ml[w][lane & 31][1] * f;
        const float* x = reinterpret_cast<const float*>(lds + w * 4 * kTile);
#pragma unroll
        for (int d = 0; d < kDim / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) core.o[0][d][i] += x[(d * 16 + i) * 64 + lane] * f;
      }
      core.m[0] = m;
    }
  }
  if (wave == 0) store_rows<T, kDim>(p, it, kv_head, core, l, 0, 32, lane);
  if (it.parts > 1) join_parts<T, kDim>(p, it, kv_head, 32);
}

}  // namespace gc
