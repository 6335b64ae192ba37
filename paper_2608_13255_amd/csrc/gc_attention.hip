// Attention over packed sequences with grouped heads.
//
// For each query row, over the keys it sees: s_j = scale q.k_j, the running
// maximum m and sum l of exp(s_j - m), out = sum exp(s_j - m) v_j / l and
// lse = m + log l, all in float32.
#include <algorithm>
#include <cmath>
#include <vector>

#include "gc_attention_core.h"

namespace gc {
namespace {

// Keys per part: a multiple of every variant's tile.
constexpr int kPartKeys = 64;
// Blocks to fill the card with: one for each of 256 compute units, two of the smaller ones.
constexpr int kCus = 256;

struct Batch {
  const int32_t *q_lens, *k_lens;
  int n_seq, group, kv_heads, causal;
};

// Keys that the rows [row0, row0 + tile) of a sequence see, at most.
int keys_seen(const Batch& b, int s, int row0, int tile) {
  if (!b.causal) return b.k_lens[s];
  const int64_t rows = (int64_t)b.q_lens[s] * b.group;
  const int64_t last = (std::min<int64_t>(rows, (int64_t)row0 + tile) - 1) / b.group;
  const int64_t n = last + b.k_lens[s] - b.q_lens[s] + 1;
  return (int)std::max<int64_t>(0, std::min<int64_t>(n, b.k_lens[s]));
}

int parts_of(int keys, int part) { return keys <= part ? 1 : (int)(((int64_t)keys + part - 1) / part); }

template <class F>
void each_tile(const Batch& b, int tile, F f) {
  int64_t q0 = 0, k0 = 0;
  for (int s = 0; s < b.n_seq; ++s) {
    const int64_t rows = (int64_t)b.q_lens[s] * b.group;
    for (int64_t r = 0; r < rows; r += tile) f(s, (int)r, (int)rows, (int)q0, (int)k0);
    q0 += b.q_lens[s], k0 += b.k_lens[s];
  }
}

// Items of a variant with parts of at most `part` keys.
int64_t items_of(const Batch& b, int tile, int part) {
  int64_t n = 0;
  each_tile(b, tile, [&](int s, int r, int, int, int) { n += parts_of(keys_seen(b, s, r, tile), part); });
  return n;
}

// The variant and the keys a part holds at most (what is longer is split).
void choose(const Batch& b, int dim, int dtype, int* kind, int* part) {
  int64_t most_rows = 0, tiles256 = 0;
  for (int s = 0; s < b.n_seq; ++s) {
    const int64_t rows = (int64_t)b.q_lens[s] * b.group;
    most_rows = std::max(most_rows, rows);
    tiles256 += (rows + 255) / 256;
  }
  if (most_rows <= 32) *kind = kAttnKeys;
  // Tiles of 256 rows read keys and values half as often (24576 x 16 x 128: 4.27 ms against 4.41 with tiles of 128); those of
  // 128 are evener where few rounds of blocks fill the card, and mask less under a causal mask (packed prompts: 709 us
  // against 721).
  else *kind = attention_has_rows256(dim, dtype) && !b.causal && tiles256 * b.kv_heads >= 2 * kCus ? kAttnRows256 : kAttnRows128;
  // the blocks that the card holds at once
  const int64_t blocks = *kind == kAttnKeys ? kCus * attention_keys_blocks(dim, dtype) : *kind == kAttnRows256 ? kCus : 2 * kCus;
  const int tile = attention_tile_rows(*kind);
  int64_t work = 0, most = 0;
  each_tile(b, tile, [&](int s, int r, int, int, int) {
    const int64_t n = keys_seen(b, s, r, tile);
    work += n, most = std::max(most, n);
  });
  // The shortest parts with which all blocks are there at once, so that they end together, but none shorter than pays for
  // joining it: 512 keys of bfloat16 (1024 tokens x 16 heads x 64: 19.2 us against 22.5 with 256), 256 of float, whose
  // products take longer, and of single tokens (8 x 1000 keys: 14.3 us against 16.4 with 512).
  const int64_t least = *kind == kAttnKeys || dtype == GC_F32 ? 256 : 512;
  int64_t low = std::max<int64_t>(work * b.kv_heads / blocks + 1, least), high = std::max(low, most);
  while (low < high) {
    const int64_t mid = (low + high) / 2;
    if (items_of(b, tile, (int)mid) * b.kv_heads <= blocks) high = mid;
    else low = mid + 1;
  }
  low = (low + kPartKeys - 1) / kPartKeys * kPartKeys;
  *part = (int)std::min<int64_t>(low, 0x7fffffc0);
}

}  // namespace
}  // namespace gc

using namespace gc;

extern "C" int gc_attention_plan(const int32_t* q_lens, const int32_t* k_lens, int n_seq, int heads, int kv_heads, int dim,
                                 int dtype, int causal, gc_attention_info* info, int32_t* items, int64_t capacity_words) {
  clear_error();
  const char* who = "gc_attention_plan";
  if (!info) return fail(GC_ERR_ARG, "%s: info is null", who);
  int rc = check_head_sizes(heads, dim, dtype, who);
  if (rc) return rc;
  if (kv_heads < 1 || heads % kv_heads) return fail(GC_ERR_SHAPE, "%s: heads=%d is not a multiple of kv_heads=%d", who, heads, kv_heads);
  if (n_seq < 0 || n_seq > (1 << 24)) return fail(GC_ERR_CAPACITY, "%s: n_seq=%d outside [0, 2^24]", who, n_seq);
  if (n_seq > 0 && (!q_lens || !k_lens)) return fail(GC_ERR_ARG, "%s: q_lens or k_lens is null", who);
  const int group = heads / kv_heads;
  int64_t total_q = 0, total_k = 0;
  for (int s = 0; s < n_seq; ++s) {
    if (q_lens[s] < 0 || k_lens[s] < 0) return fail(GC_ERR_SHAPE, "%s: sequence %d has lengths %d and %d", who, s, q_lens[s], k_lens[s]);
    total_q += q_lens[s];
    total_k += k_lens[s];
    if ((int64_t)q_lens[s] * group > 0x7fffffffLL - GC_MAX_HEADS) return fail(GC_ERR_CAPACITY, "%s: sequence %d has over 2^31 query rows", who, s);
  }
  if (total_q > 0x7fffffffLL || total_k > 0x7fffffffLL - 1024) return fail(GC_ERR_CAPACITY, "%s: over 2^31-1 tokens", who);
  const Batch b = {q_lens, k_lens, n_seq, group, kv_heads, causal};
  int kind, part;
  choose(b, dim, dtype, &kind, &part);
  const int tile = attention_tile_rows(kind);
  int64_t n_items = 0, n_slots = 0, n_groups = 0;
  each_tile(b, tile, [&](int s, int r, int, int, int) {
    const int n = parts_of(keys_seen(b, s, r, tile), part);
    n_items += n;
    if (n > 1) n_slots += n, ++n_groups;
  });
  if (n_items * kv_heads > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: over 2^31-1 blocks", who);
  std::memset(info, 0, sizeof(*info));
  info->heads = heads, info->kv_heads = kv_heads, info->dim = dim, info->dtype = dtype, info->causal = causal != 0;
  info->n_seq = n_seq, info->total_q = (int32_t)total_q, info->total_k = (int32_t)total_k;
  info->kind = kind, info->tile_rows = tile, info->n_items = (int32_t)n_items;
  info->n_slots = (int32_t)n_slots, info->n_groups = (int32_t)n_groups;
  info->workspace_bytes = n_slots * kv_heads * tile * (int64_t)(attention_padded_dim(dim) + 2) * 4;
  if (!items) return GC_OK;
  if (capacity_words < n_items * GC_ATTENTION_ITEM_WORDS)
    return fail(GC_ERR_CAPACITY, "%s: %lld words for %lld items of %d", who, (long long)capacity_words, (long long)n_items, GC_ATTENTION_ITEM_WORDS);
  AttentionItem* it = reinterpret_cast<AttentionItem*>(items);
  int32_t slot = 0, group_id = 0;
  each_tile(b, tile, [&](int s, int r, int rows, int q0, int k0) {
    const int keys = keys_seen(b, s, r, tile), n = parts_of(keys, part);
    // the parts as equal as whole tiles of keys allow
    const int64_t step = (((int64_t)keys + n - 1) / n + kPartKeys - 1) / kPartKeys * kPartKeys;
    for (int i = 0; i < n; ++i) {
      const int begin = (int)std::min<int64_t>(i * step, keys), end = (int)std::min<int64_t>((i + 1) * step, keys);
      *it++ = AttentionItem{q0, rows, r, k0, begin, i + 1 == n ? keys : end, k_lens[s] - q_lens[s] + 1, k_lens[s],
                            n > 1 ? slot + i : -1, n > 1 ? slot : -1, n, n > 1 ? group_id : -1};
    }
    if (n > 1) slot += n, ++group_id;
  });
  // the longest first: what is left at the end is short
  AttentionItem* first = reinterpret_cast<AttentionItem*>(items);
  std::stable_sort(first, it, [](const AttentionItem& x, const AttentionItem& y) { return x.k_end - x.k_begin > y.k_end - y.k_begin; });
  return GC_OK;
}

extern "C" int gc_attention(const gc_heads* q, const gc_heads* k, const gc_heads* v, const gc_heads* out, float* lse,
                            const gc_attention_info* info, const int32_t* items, double scale, void* workspace,
                            size_t ws_bytes, hipStream_t stream) {
  clear_error();
  const char* who = "gc_attention";
  if (!info) return fail(GC_ERR_ARG, "%s: info is null", who);
  int rc = check_head_sizes(info->heads, info->dim, info->dtype, who);
  if (rc) return rc;
  if (info->kv_heads < 1 || info->heads % info->kv_heads || info->kind < 0 || info->kind >= kAttnKinds ||
      (info->kind == kAttnRows256 && !attention_has_rows256(info->dim, info->dtype)) || info->tile_rows != attention_tile_rows(info->kind) ||
      info->n_items < 0 || info->total_q < 0 || info->total_k < 0 || info->n_slots < 0 || info->n_groups < 0 ||
      info->workspace_bytes < (int64_t)info->n_slots * info->kv_heads * info->tile_rows * (attention_padded_dim(info->dim) + 2) * 4)
    return fail(GC_ERR_ARG, "%s: info is not gc_attention_plan's", who);
  if (!(scale > 0.0) || !std::isfinite(scale)) return fail(GC_ERR_ARG, "%s: scale must be finite and above 0", who);
  if (info->n_items == 0) return GC_OK;
  if (!items) return fail(GC_ERR_ARG, "%s: items is null", who);
  if (!aligned16(items) || (reinterpret_cast<uintptr_t>(lse) & 3) || (workspace && !aligned16(workspace)))
    return fail(GC_ERR_ALIGN, "%s: items, lse or workspace misaligned", who);
  if (info->workspace_bytes > 0 && !workspace) return fail(GC_ERR_ARG, "%s: workspace is null", who);
  if (ws_bytes < (size_t)info->workspace_bytes)
    return fail(GC_ERR_CAPACITY, "%s: workspace of %zu bytes is below the %lld required", who, ws_bytes, (long long)info->workspace_bytes);
  const int dtype = info->dtype, dim = info->dim;
  if ((rc = check_heads(q, dtype, "q", who)) || (rc = check_heads(out, dtype, "out", who)) ||
      (rc = check_heads_out(*out, info->total_q, info->heads, dim, "out", who)))
    return rc;
  if (info->total_k > 0 && ((rc = check_heads(k, dtype, "k", who)) || (rc = check_heads(v, dtype, "v", who)))) return rc;
  // the range of a tile's buffer ends at its sequence's last key: tokens may not share memory
  if (info->total_k > 1 && (k->token_stride < dim || v->token_stride < dim))
    return fail(GC_ERR_SHAPE, "%s: the token strides of k and v must be at least dim=%d", who, dim);
  const int64_t es = dtype_bytes(dtype);
  const size_t out_bytes = (size_t)((info->total_q - 1) * out->token_stride + (info->heads - 1) * out->head_stride + dim) * es;
  const size_t lse_bytes = lse ? (size_t)info->heads * info->total_q * 4 : 0;
  const size_t item_bytes = (size_t)info->n_items * sizeof(AttentionItem);
  const gc_heads* in[3] = {q, k, v};
  for (int i = 0; i < 3; ++i) {
    const int64_t t = i ? info->total_k : info->total_q;
    const int h = i ? info->kv_heads : info->heads;
    if (t == 0) continue;
    const size_t bytes = (size_t)((t - 1) * in[i]->token_stride + (h - 1) * in[i]->head_stride + dim) * es;
    if (heads_overlap(*in[i], t, h, *out, info->total_q, info->heads, dim, dtype) || overlaps(in[i]->data, bytes, lse, lse_bytes) ||
        overlaps(in[i]->data, bytes, workspace, (size_t)info->workspace_bytes))
      return fail(GC_ERR_ALIAS, "%s: out, lse or workspace overlaps %s", who, i == 0 ? "q" : i == 1 ? "k" : "v");
  }
  if (overlaps(out->data, out_bytes, lse, lse_bytes) || overlaps(out->data, out_bytes, items, item_bytes) ||
      overlaps(lse, lse_bytes, items, item_bytes) || overlaps(workspace, (size_t)info->workspace_bytes, out->data, out_bytes) ||
      overlaps(workspace, (size_t)info->workspace_bytes, lse, lse_bytes) || overlaps(workspace, (size_t)info->workspace_bytes, items, item_bytes))
    return fail(GC_ERR_ALIAS, "%s: out, lse, items and workspace overlap", who);
  AttentionArgs p = {};
  p.q = q->data, p.q_token = q->token_stride, p.q_head = q->head_stride;
  if (info->total_k > 0) {
    p.k = k->data, p.k_token = k->token_stride, p.k_head = k->head_stride;
    p.v = v->data, p.v_token = v->token_stride, p.v_head = v->head_stride;
  }
  p.out = out->data, p.o_token = out->token_stride, p.o_head = out->head_stride;
  p.lse = lse;
  p.items = reinterpret_cast<const AttentionItem*>(items);
  p.heads = info->heads, p.kv_heads = info->kv_heads, p.group = info->heads / info->kv_heads, p.dim = dim;
  p.total_q = info->total_q, p.total_k = info->total_k;
  p.causal = info->causal;
  p.scale = (float)scale;
  if (info->n_slots > 0) p.partial = reinterpret_cast<float*>(workspace);
  const unsigned blocks = (unsigned)(info->n_items * info->kv_heads);
  const bool known = dtype == GC_F32 ? launch_attention_f32(p, info->kind, blocks, stream)
                                     : launch_attention_bf16(p, info->kind, blocks, stream);
  if (!known) return fail(GC_ERR_SHAPE, "%s: no kernel for dim=%d", who, dim);
  return after_launch(stream, who);
}
