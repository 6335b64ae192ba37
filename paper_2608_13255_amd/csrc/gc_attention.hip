// Attention over packed sequences with grouped heads.
//
// For each query row, over the keys it sees: s_j = scale q.k_j, the running
// maximum m and sum l of exp(s_j - m), out = sum exp(s_j - m) v_j / l and
// lse = m + log l, all in float32 (bfloat16 heads: the weights are rounded to
// bfloat16 for the second product, and the results on their way out).
//
// A call cannot do without reading q, k and v and writing out once, and 4 dim
// operations a head and visible pair: single tokens are bound by the read,
// everything else by the operations.  Measured, us, with the time of the
// bound at a large read's 7.0 TB/s or a large product's 1378 (bfloat16) and
// 153 (float32) TFLOP/s (boxes differ by up to 7 %: the slowest took 152, 527, 712 and 4311 for the last four):
//   8 single tokens, 32 heads on 8 of 128, 495 MB of keys and values     90   71
//   1024 + 1 + 517 + 770 tokens, 8 heads of 64, float32                  51   25
//   10403 tokens in 4 sequences, 16 heads of 64, among themselves       145   83
//   the same over 31070 keys, 16 heads of 80 (worked on as 96)          504  308
//   15427 causal tokens in 7 sequences, 32 heads on 8 of 128            672  527
//   24576 tokens, 16 heads of 128                                      4048 3592
#include <algorithm>
#include <cmath>
#include <exception>
#include <functional>
#include <queue>
#include <vector>

#include "gc_attention_core.h"

namespace gc {
namespace {

// Keys per part: a multiple of every variant's tile.
constexpr int kPartKeys = 64;
// Compute units.
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

// What a variant takes, in microseconds, from timings on a full card: a block
// alone on its compute unit goes through `rate` keys a microsecond, two that
// share one through `share` times as many together; a block's first loads
// and its results take kBlockTime.  (kAttnKeys by the bytes that it reads, also in float32 above 64 channels, where its
// products take longer: its parts then differ in length alone.)
struct Cost {
  int kind;
  double rate, share;
};
constexpr double kBlockTime = 3.0;

Cost cost_of(int kind, int dim, int dtype) {
  const int padded = std::max(64, attention_padded_dim(dim));
  if (kind == kAttnKeys) return {kind, 45.0 * 256 / (padded * dtype_bytes(dtype) / 2.0) / 2, 1.0};
  if (dtype == GC_F32) return {kind, 14.6 * 64 / padded, padded <= 96 ? 1.3 : 1.0};
  if (kind == kAttnRows256) return {kind, std::min(57.0, 4400.0 / padded), 1.0};
  return {kind, std::min(85.0, 6400.0 / padded), padded <= 128 ? 1.3 : 1.0};
}

// The time of the tiles' keys in parts of at most `part`: parts are dealt, the
// longest first, each to the compute unit with least to do (a kv head's
// share of the units: all heads do the same), and joined in a launch of
// its own, which takes 8 us, a quarter for each of a tile's parts, and the partial results' way out and back.
double time_of(const std::vector<int>& tiles, int part, const Cost& c, int kv_heads, int dim) {
  const size_t lanes = (size_t)std::max(1, kCus / kv_heads);
  std::vector<int> pieces;
  int64_t slots = 0;
  int most = 1;
  for (int keys : tiles) {
    const int n = parts_of(keys, part);
    for (int i = 0; i < n; ++i) pieces.push_back((keys + n - 1) / n);
    if (n > 1) slots += n, most = std::max(most, n);
  }
  std::sort(pieces.begin(), pieces.end(), std::greater<int>());
  std::priority_queue<double, std::vector<double>, std::greater<double>> busy;
  double last = 0;
  for (int keys : pieces) {
    double t = keys / c.rate + kBlockTime;
    const bool first = busy.size() < lanes;
    if (!first) t += busy.top(), busy.pop();
    busy.push(t);
    last = std::max(last, first ? t : t / c.share);
  }
  const double bytes = 4.0 * slots * kv_heads * attention_tile_rows(c.kind) * attention_padded_dim(dim);
  return last + (slots ? 8.0 + 0.25 * most + 2 * bytes / 5e6 : 0.0);
}

// The variant and the keys a part holds at most (what is longer is split):
// single tokens and other sequences of at most 32 rows share a block's
// rows among its waves' keys; else 128 or 256 rows a block, whichever takes
// less time.  256 rows read each tile of keys half as often, 128 leave less
// over at a sequence's and at the launch's end.  256 against 128: 24576 tokens
// x 16 heads x 128 4.05 ms and 4.54, 16384 causal x 8 x 128 491 us and 562,
// 4096 x 16 x 64 83 and 89; 2048 x 16 x 64 36 and 27, 6000 x 12 x 96 228 and
// 219, 4096 causal x 8 x 128 64 and 60.  Parts: 160 rows over 9000 keys 22 us
// in 29 against 150 whole; 2048 x 16 x 64 27 whole against 35 in two.
void choose(const Batch& b, int dim, int dtype, int* kind, int* part) {
  int64_t most_rows = 0;
  for (int s = 0; s < b.n_seq; ++s) most_rows = std::max(most_rows, (int64_t)b.q_lens[s] * b.group);
  double best = 0;
  *part = 0x7fffffc0;
  *kind = most_rows <= 32 ? kAttnKeys : kAttnRows128;
  for (int k = 0; k < kAttnKinds; ++k) {
    if ((k == kAttnKeys) != (most_rows <= 32) || (k == kAttnRows256 && !attention_has_rows256(dim, dtype))) continue;
    const Cost c = cost_of(k, dim, dtype);
    const int tile = attention_tile_rows(k);
    std::vector<int> tiles;
    int64_t work = 0;
    int most = 0;
    each_tile(b, tile, [&](int s, int r, int, int, int) {
      const int n = keys_seen(b, s, r, tile);
      tiles.push_back(n), work += n, most = std::max(most, n);
    });
    const int64_t lanes = std::max(1, kCus / b.kv_heads);
    // many rounds of whole tiles are even enough: only their sum counts
    const bool many = (int64_t)tiles.size() >= 16 * lanes;
    const double whole = many ? (work / c.rate + tiles.size() * kBlockTime) / lanes / c.share : time_of(tiles, 0x7fffffc0, c, b.kv_heads, dim);
    if (best == 0 || whole < best) best = whole, *kind = k, *part = 0x7fffffc0;
    if (many || most <= kPartKeys) continue;
    for (const double rounds : {0.5, 0.75, 0.9, 1.0, 1.1, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 4.0}) {
      const int64_t keys = ((int64_t)((double)work / lanes / rounds) / kPartKeys + 1) * kPartKeys;
      if (keys >= most) continue;
      const double t = time_of(tiles, (int)keys, c, b.kv_heads, dim);
      if (t < best) best = t, *kind = k, *part = (int)keys;
    }
  }
}

}  // namespace
}  // namespace gc

using namespace gc;

namespace {

int make_plan(const int32_t* q_lens, const int32_t* k_lens, int n_seq, int heads, int kv_heads, int dim, int dtype,
              int causal, gc_attention_info* info, int32_t* items, int64_t capacity_words, const char* who) {
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
  if (n_items > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: over 2^31-1 items", who);
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

}  // namespace

extern "C" int gc_attention_plan(const int32_t* q_lens, const int32_t* k_lens, int n_seq, int heads, int kv_heads, int dim,
                                 int dtype, int causal, gc_attention_info* info, int32_t* items, int64_t capacity_words) {
  clear_error();
  const char* who = "gc_attention_plan";
  try {
    return make_plan(q_lens, k_lens, n_seq, heads, kv_heads, dim, dtype, causal, info, items, capacity_words, who);
  } catch (const std::exception&) {   // the lists of tiles and parts
    return fail(GC_ERR_CAPACITY, "%s: no host memory for %d sequences", who, n_seq);
  }
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
  // (a scale that is 0 in float32 would make the masked scores' -inf NaN)
  if (!((float)scale > 0.f) || !std::isfinite((float)scale * kLog2e))
    return fail(GC_ERR_ARG, "%s: scale=%g must be finite and above 0 in float32", who, scale);
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
  p.kv_heads = info->kv_heads, p.group = info->heads / info->kv_heads, p.dim = dim;
  p.total_q = info->total_q;
  p.causal = info->causal;
  p.scale = (float)scale;
  if (info->n_slots > 0) p.partial = reinterpret_cast<float*>(workspace);
  const int most = std::max(1, kMostBlocks / info->kv_heads);
  for (const bool join : {false, true}) {
    if (join && !p.partial) break;
    for (int i = 0; i < info->n_items; i += std::min(most, info->n_items - i)) {
      p.items = reinterpret_cast<const AttentionItem*>(items) + i;
      const unsigned blocks = (unsigned)(std::min(most, info->n_items - i) * info->kv_heads);
      const bool known = dtype == GC_F32 ? launch_attention_f32(p, info->kind, join, blocks, stream)
                                         : launch_attention_bf16(p, info->kind, join, blocks, stream);
      if (!known) return fail(GC_ERR_SHAPE, "%s: no kernel for dim=%d", who, dim);
    }
  }
  return after_launch(stream, who);
}
