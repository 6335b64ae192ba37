// Attention kernels for bfloat16 heads.
#include "gc_attention_kernels.h"

namespace gc {

namespace {

template <int kDim>
void launch(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream) {
  constexpr int kWaves = attention_keys_waves(kDim, 2);
  if (join) return launch_join<uint16_t, kDim>(p, attention_tile_rows(kind), blocks, stream);
  // Keys a tile: 64 where the registers hold their scores beside the output (24576 tokens x 16 heads x 128 4.11 ms
  // against 4.22 with 32) and two blocks of four waves fit a compute unit's LDS.
  constexpr int kBlocks = kDim <= 128 ? 2 : 1, kBlocks128 = kDim <= 96 ? 2 : 1, kPerSimd = kDim <= 128 ? 2 : 1;
  if constexpr (kDim <= 128) {
    if (kind == kAttnRows256) {
      hipLaunchKernelGGL((k_attention_rows<kDim, kBlocks, 8, 2>), dim3(blocks), dim3(512), 0, stream, p);
    }
  }
  if (kind == kAttnKeys) hipLaunchKernelGGL((k_attention_keys<uint16_t, kDim, kWaves>), dim3(blocks), dim3(64 * kWaves), 0, stream, p);
  else if (kind == kAttnRows128) hipLaunchKernelGGL((k_attention_rows<kDim, kBlocks128, 4, kPerSimd>), dim3(blocks), dim3(256), 0, stream, p);
}

}  // namespace

bool launch_attention_bf16(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream) {
  switch (attention_padded_dim(p.dim)) {
    case 32: launch<32>(p, kind, join, blocks, stream); return true;
    case 64: launch<64>(p, kind, join, blocks, stream); return true;
    case 96: launch<96>(p, kind, join, blocks, stream); return true;
    case 128: launch<128>(p, kind, join, blocks, stream); return true;
    case 192: launch<192>(p, kind, join, blocks, stream); return true;
    case 256: launch<256>(p, kind, join, blocks, stream); return true;
  }
  return false;
}

}  // namespace gc
