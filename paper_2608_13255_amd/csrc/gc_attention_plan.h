// The work of a batch of packed sequences, laid out on the host: items of
// query rows, as the kernels read them.
#pragma once

#include "gc_heads.h"

namespace gc {

// One item: rows [row0, row0 + tile) of one sequence over its keys
// [k_begin, k_end), for every kv head.  Row r is query token r / group, head
// r % group of the kv head's group, so the heads that share keys share a tile.
struct AttentionItem {
  int32_t q_token0;   // the sequence's first query token
  int32_t rows;       // its rows: query tokens * group
  int32_t row0;
  int32_t k_token0;   // the sequence's first key token
  int32_t k_begin, k_end;
  int32_t reach;      // token i sees keys [0, i + reach), clamped to k_len
  int32_t k_len;
  int32_t slot;       // this part's partial result, -1: the item holds all of its rows' keys
  int32_t slot0;      // the tile's first part
  int32_t parts;      // its number of parts
  int32_t group_id;   // its number among the split tiles (host: what info counts as n_groups)
};
static_assert(sizeof(AttentionItem) == GC_ATTENTION_ITEM_WORDS * 4, "item words");

// Kernel variants (gc_attention_info.kind) and their rows an item.
enum AttentionKind { kAttnRows256 = 0, kAttnRows128 = 1, kAttnKeys = 2, kAttnKinds = 3 };
inline int attention_tile_rows(int kind) { return kind == kAttnRows256 ? 256 : kind == kAttnRows128 ? 128 : 32; }

// Head dims are padded to the next of these in LDS and registers.
inline int attention_padded_dim(int dim) {
  return dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256;
}

// Whether two waves' rows a SIMD fit the registers with eight waves a block.
inline bool attention_has_rows256(int dim, int dtype) { return dtype == GC_BF16 && attention_padded_dim(dim) <= 128; }

// The waves of a block of kAttnKeys: two tiles of 32 keys and two of values
// for each of them, in at most 128 of a compute unit's 160 KiB of LDS.
constexpr int attention_keys_waves(int padded, int bytes) {
  return padded * bytes <= 256 ? 4 : padded * bytes <= 512 ? 2 : 1;
}

struct AttentionArgs;
// Blocks of a launch: its threads (at most 512 a block) are counted in 32 bits.
constexpr int kMostBlocks = 1 << 22;
// Launches of one storage type: the items' results, or (join) those of split rows from their parts.
// false: no such variant.
bool launch_attention_bf16(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream);
bool launch_attention_f32(const AttentionArgs& p, int kind, bool join, unsigned blocks, hipStream_t stream);

}  // namespace gc
