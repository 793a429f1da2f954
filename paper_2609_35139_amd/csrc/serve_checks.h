// Host-side checks shared by the entry points that work on a paged cache
// (internal to the library).
#pragma once
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "serve.h"
#include "validate.h"

namespace cr {

constexpr int64_t kMostTokens = ((int64_t)1 << 31) - 256;

// The batch as the host sees it.
struct Batch {
  int64_t n_tokens = 0;
  int64_t most = 0;              // queries of the longest sequence
  const int32_t* off = nullptr;  // null: every sequence has n_tokens / n_seqs queries
};

inline cr_status check_cache(const cr_kv_layout* l) {
  if (l->n_layers < 1 || l->n_kv_heads < 1 || l->head_dim < 32 || l->head_dim > 256 ||
      l->head_dim % 32)
    return CR_ERR_DIMS;
  return check_dtype(l);
}

// The offsets and the table's extent (no device memory is read).
inline cr_status check_batch(const cr_sequences* q, Batch* b) {
  if (q->n_seqs < 1) return CR_ERR_OFFSETS;
  if (!q->query_offsets) {
    b->n_tokens = q->n_seqs;
    b->most = 1;
  } else {
    const int32_t* o = q->query_offsets;
    if (o[0] != 0) return CR_ERR_OFFSETS;
    bool same = true;
    for (int s = 0; s < q->n_seqs; ++s) {
      if (o[s + 1] < o[s]) return CR_ERR_OFFSETS;
      b->most = std::max<int64_t>(b->most, (int64_t)o[s + 1] - o[s]);
      same = same && o[s + 1] - o[s] == o[1];
    }
    b->n_tokens = o[q->n_seqs];
    if (!same) b->off = o;
  }
  if (b->n_tokens >= kMostTokens) return CR_ERR_DIMS;
  if (q->block_size < 1 || q->block_size > 1024 || (q->block_size & (q->block_size - 1)) ||
      q->max_blocks < 1 || (int64_t)q->max_blocks * q->block_size >= kMostTokens)
    return CR_ERR_LAYOUT;
  return CR_OK;
}

// A [n][heads][head_dim] operand; written ones must not overlap themselves.
inline cr_status check_rows(const cr_rows* r, int64_t n, int64_t heads, int64_t head_dim, bool written) {
  if (!r->data && n > 0) return CR_ERR_NULL;
  if (!aligned(r->data, 16)) return CR_ERR_LAYOUT;
  const int64_t st[2] = {r->stride_token, r->stride_head}, ext[2] = {n, heads};
  Dims dims;
  dims.push_back({1, head_dim});
  if (n == 0) return CR_OK;   // no element is addressed
  int64_t reach = 0;
  for (int i = 0; i < 2; ++i) {
    if (st[i] < 0 || st[i] % 8) return CR_ERR_LAYOUT;
    int64_t span;
    if (__builtin_mul_overflow(st[i], ext[i] - 1, &span) ||
        __builtin_add_overflow(reach, span, &reach) || reach >= (int64_t)1 << 62)
      return CR_ERR_LAYOUT;
    if (ext[i] > 1) dims.push_back({st[i], ext[i]});
  }
  return written ? check_injective(dims) : CR_OK;
}

// The block geometry; the kernels take the bytes between a block's rows in 32 bits.
inline cr_status check_blocks(const cr_kv_layout* l, const cr_sequences* q) {
  const cr_status st = check_page_strides(l, q->block_size, q->n_blocks, q->stride_block);
  if (st != CR_OK) return st;
  if (q->block_size > 1 && l->stride_token >= ((int64_t)1 << 32) / (int64_t)esize(l->dtype))
    return CR_ERR_LAYOUT;
  return CR_OK;
}

inline PagedSeqs paged(const cr_kv_layout* l, const cr_sequences* q) {
  PagedSeqs p{};
  p.token = l->stride_token;
  p.head = l->stride_head;
  p.block = q->stride_block;
  p.shift = log2_int(q->block_size);
  p.n_blocks = q->n_blocks;
  p.max_blocks = q->max_blocks;
  p.max_len = q->max_blocks * q->block_size;
  p.n_seqs = q->n_seqs;
  p.table = q->block_table;
  p.lens = q->kv_lens;
  return p;
}

// Address of component c (0 K, 1 V) of a layer.
inline const char* component(const void* kv, const cr_kv_layout* l, int layer, int c) {
  return static_cast<const char*>(kv) +
         ((int64_t)layer * l->stride_layer + (int64_t)c * l->stride_kv) * (int64_t)esize(l->dtype);
}

// The heads of a call and the batch they belong to.
inline cr_status check_attend(const cr_kv_layout* l, const cr_sequences* q, int n_heads, int shared,
                       Batch* b) {
  cr_status st = check_cache(l);
  if (st != CR_OK) return st;
  st = check_batch(q, b);
  if (st != CR_OK) return st;
  if (n_heads < 1 || n_heads > kMaxQueryHeads || n_heads % l->n_kv_heads) return CR_ERR_DIMS;
  if (b->n_tokens * n_heads >= kMostTokens) return CR_ERR_DIMS;
  if (shared < 0 || shared > q->max_blocks * q->block_size) return CR_ERR_DIMS;
  return CR_OK;
}

// The options of a score.
inline cr_status check_scores(const cr_attend_options& o, int n_heads) {
  if (!(o.scale >= 0.f) || !std::isfinite(o.scale) || !(o.softcap >= 0.f) ||
      !std::isfinite(o.softcap))
    return CR_ERR_DIMS;
  for (int h = 0; o.slopes && h < n_heads; ++h)
    if (!std::isfinite(o.slopes[h])) return CR_ERR_DIMS;
  return CR_OK;
}

// The factors of cr_attend_options in the kernels' units (A: AttendArgs or
// WeighArgs).
template <typename A>
inline void set_scores(A& a, const cr_attend_options& o, int n_heads) {
  const double scale = o.scale > 0.f ? o.scale : 1.0 / std::sqrt((double)a.head_dim);
  const double log2e = 1.4426950408889634;
  // (infinite factors would make NaN of a score or a distance of 0)
  auto factor = [](double x) { return (float)std::clamp(x, -(double)FLT_MAX, (double)FLT_MAX); };
  a.scale_log2 = factor(scale * log2e);
  if (o.softcap > 0.f) {
    a.cap_log2 = factor(o.softcap * log2e);
    a.scale_over_cap = factor(scale / o.softcap);
  }
  if (o.slopes) {
    a.bias = 1;
    for (int h = 0; h < n_heads; ++h) a.slopes_log2[h] = factor(o.slopes[h] * log2e);
  }
}

}  // namespace cr
