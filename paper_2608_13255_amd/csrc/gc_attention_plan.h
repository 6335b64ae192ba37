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
  int32_t group_id;   // its counter
};
static_assert(sizeof(AttentionItem) == GC_ATTENTION_ITEM_WORDS * 4, "item words");

// kernel variants (gc_attention_info.kind)
constexpr int kAttnRows = 0;

}  // namespace gc
