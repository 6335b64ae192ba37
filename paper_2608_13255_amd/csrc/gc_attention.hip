// Attention over packed sequences with grouped heads.
//
// For each query row, over the keys it sees: s_j = scale q.k_j, the running
// maximum m and sum l of exp(s_j - m), out = sum exp(s_j - m) v_j / l and
// lse = m + log l, all in float32.
#include <algorithm>
#include <cmath>
#include <vector>

#include "gc_attention_plan.h"

namespace gc {
namespace {

struct AttentionArgs {
  const void *q, *k, *v;
  void* out;
  float* lse;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  const AttentionItem* items;
  int heads, kv_heads, group, dim;
  int total_q, total_k;
  int causal;
  float scale;
};

constexpr int kSimpleBlock = 256;
constexpr int kSimpleRows = 32;

// One wave takes a row at a time: its 64 lanes score 64 keys, then hold up to
// four channels each of the weighted sum of the values.
template <class T>
__global__ __launch_bounds__(kSimpleBlock) void k_attention_rows(const AttentionArgs p) {
  __shared__ float qs[kSimpleBlock / 64][GC_MAX_HEAD_DIM];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int kvh = blockIdx.x % p.kv_heads;
  const AttentionItem it = p.items[blockIdx.x / p.kv_heads];
  const int last = it.row0 + kSimpleRows < it.rows ? it.row0 + kSimpleRows : it.rows;
  for (int r = it.row0 + wave; r < last; r += kSimpleBlock / 64) {
    const int tok = r / p.group, head = kvh * p.group + r % p.group;
    const int64_t qt = (int64_t)it.q_token0 + tok;
    const T* q = (const T*)p.q + qt * p.q_token + head * p.q_head;
    for (int d = lane * 2; d < p.dim; d += 128) {
      float x[2];
      load_heads<2>(q + d, x);
      qs[wave][d] = x[0], qs[wave][d + 1] = x[1];
    }
    __builtin_amdgcn_wave_barrier();
    int n = it.k_len;
    if (p.causal) n = tok + it.reach < n ? tok + it.reach : n;
    float m = -__builtin_inff(), l = 0.f, acc[4] = {};
    for (int j0 = 0; j0 < n; j0 += 64) {
      const int j = j0 + lane;
      float s = -__builtin_inff();
      if (j < n) {
        const T* k = (const T*)p.k + ((int64_t)it.k_token0 + j) * p.k_token + kvh * p.k_head;
        float dot = 0.f;
        for (int d = 0; d < p.dim; d += 4) {
          float x[4];
          load_heads<4>(k + d, x);
          for (int i = 0; i < 4; ++i) dot = __builtin_fmaf(x[i], qs[wave][d + i], dot);
        }
        s = dot * p.scale;
      }
      float mx = s;
      for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
      const float mn = fmaxf(m, mx);
      const float ms = mn == -__builtin_inff() ? 0.f : mn;
      const float w = expf(s - ms), f = expf(m - ms);
      m = mn;
      float sum = w;
      for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
      l = l * f + sum;
      for (int i = 0; i < 4; ++i) acc[i] *= f;
      const int c = n - j0 < 64 ? n - j0 : 64;
      for (int jj = 0; jj < c; ++jj) {
        const float wj = __shfl(w, jj);
        const T* v = (const T*)p.v + ((int64_t)it.k_token0 + j0 + jj) * p.v_token + kvh * p.v_head;
        for (int i = 0; i < 4; i += 2) {
          const int d = 2 * lane + 64 * i;
          if (d < p.dim) {
            float x[2];
            load_heads<2>(v + d, x);
            acc[i] = __builtin_fmaf(wj, x[0], acc[i]);
            acc[i + 1] = __builtin_fmaf(wj, x[1], acc[i + 1]);
          }
        }
      }
    }
    // l > 0, or NaN scores: a row without a key or with scores of -inf alone is 0
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    T* o = (T*)p.out + qt * p.o_token + head * p.o_head;
    for (int i = 0; i < 4; i += 2) {
      const int d = 2 * lane + 64 * i;
      if (d < p.dim) {
        const float x[2] = {none ? 0.f : acc[i] * inv, none ? 0.f : acc[i + 1] * inv};
        store_heads<2>(o + d, x);
      }
    }
    if (p.lse && lane == 0) p.lse[(int64_t)head * p.total_q + qt] = none ? -__builtin_inff() : m + logf(l);
  }
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
  int64_t total_q = 0, total_k = 0, n_items = 0;
  const int tile = kSimpleRows;
  for (int s = 0; s < n_seq; ++s) {
    if (q_lens[s] < 0 || k_lens[s] < 0) return fail(GC_ERR_SHAPE, "%s: sequence %d has lengths %d and %d", who, s, q_lens[s], k_lens[s]);
    total_q += q_lens[s];
    total_k += k_lens[s];
    if ((int64_t)q_lens[s] * group > 0x7fffffffLL - GC_MAX_HEADS) return fail(GC_ERR_CAPACITY, "%s: sequence %d has over 2^31 query rows", who, s);
    n_items += ((int64_t)q_lens[s] * group + tile - 1) / tile;
  }
  if (total_q > 0x7fffffffLL || total_k > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: over 2^31-1 tokens", who);
  if (n_items * kv_heads > 0x7fffffffLL) return fail(GC_ERR_CAPACITY, "%s: over 2^31-1 blocks", who);
  std::memset(info, 0, sizeof(*info));
  info->heads = heads, info->kv_heads = kv_heads, info->dim = dim, info->dtype = dtype, info->causal = causal != 0;
  info->n_seq = n_seq, info->total_q = (int32_t)total_q, info->total_k = (int32_t)total_k;
  info->kind = kAttnRows, info->tile_rows = tile, info->n_items = (int32_t)n_items;
  if (!items) return GC_OK;
  if (capacity_words < n_items * GC_ATTENTION_ITEM_WORDS)
    return fail(GC_ERR_CAPACITY, "%s: %lld words for %lld items of %d", who, (long long)capacity_words, (long long)n_items, GC_ATTENTION_ITEM_WORDS);
  AttentionItem* it = reinterpret_cast<AttentionItem*>(items);
  int64_t q0 = 0, k0 = 0;
  for (int s = 0; s < n_seq; ++s) {
    const int rows = q_lens[s] * group;
    for (int r = 0; r < rows; r += tile)
      *it++ = AttentionItem{(int32_t)q0, rows, r, (int32_t)k0, 0, k_lens[s], k_lens[s] - q_lens[s] + 1, k_lens[s], -1, -1, 1, -1};
    q0 += q_lens[s], k0 += k_lens[s];
  }
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
  if (info->kv_heads < 1 || info->heads % info->kv_heads || info->kind != kAttnRows || info->tile_rows != kSimpleRows ||
      info->n_items < 0 || info->total_q < 0 || info->total_k < 0 || info->workspace_bytes < 0)
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
  const dim3 grid((unsigned)(info->n_items * info->kv_heads));
  if (dtype == GC_F32) hipLaunchKernelGGL(k_attention_rows<float>, grid, dim3(kSimpleBlock), 0, stream, p);
  else hipLaunchKernelGGL(k_attention_rows<uint16_t>, grid, dim3(kSimpleBlock), 0, stream, p);
  return after_launch(stream, who);
}
