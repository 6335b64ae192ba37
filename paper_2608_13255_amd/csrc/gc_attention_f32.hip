// Attention kernels for float32 heads.
#include "gc_attention_kernels.h"

namespace gc {
namespace {

template <int kDim>
void launch(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream) {
  constexpr int kWaves = attention_keys_waves(kDim, 4);
  if (join) return launch_join<float, kDim>(p, attention_tile_rows(kind), blocks, stream);
  if (kind == kAttnKeys) hipLaunchKernelGGL((k_attention_keys<float, kDim, kWaves>), dim3(blocks), dim3(64 * kWaves), 0, stream, p);
  else if (kind == kAttnRows128) hipLaunchKernelGGL((k_attention_rows_f32<kDim, kDim <= 96 ? 2 : 1>), dim3(blocks), dim3(256), 0, stream, p);
}

}  // namespace

bool launch_attention_f32(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream) {
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
