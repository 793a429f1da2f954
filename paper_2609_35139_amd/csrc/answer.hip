// C ABI of keeping an answer going: validation and the launches of
// cr_weigh_keys, cr_choose_slots, cr_compact_kv and cr_sample.  See
// include/cacherepair.h.
#include "answer.h"

#include "../../include/cacherepair.h"
#include "profile.h"
#include "rules.h"
#include "serve_checks.h"

namespace {

using namespace cr;   // the helpers of validate.h, serve_checks.h and profile.h

constexpr int64_t kMostSlots = (int64_t)1 << 30;   // of a sequence's weights, or in its list

// Lengths that a call writes, or reads beside kv_lens, in those it only reads.
bool lens_overlap(const int32_t* a, const int32_t* b, int n) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && (x < y ? y - x : x - y) < (uintptr_t)n * 4;
}

// The weights' rows, one of the table's slots for each layer, sequence and head.
cr_status check_weights(const cr_key_weights* w, int n_layers, int n_heads, const cr_sequences* q) {
  if (!w->data) return CR_ERR_NULL;
  if (!aligned(w->data, 4)) return CR_ERR_LAYOUT;
  const int64_t st[3] = {w->stride_layer, w->stride_seq, w->stride_head};
  const int64_t ext[3] = {n_layers, q->n_seqs, n_heads};
  Dims dims;
  dims.push_back({1, (int64_t)q->max_blocks * q->block_size});
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return CR_ERR_LAYOUT;
    if (ext[i] > 1) dims.push_back({st[i], ext[i]});
  }
  return check_injective(dims);
}

SlotWeights slot_weights(const cr_key_weights* w) {
  return w ? SlotWeights{w->data, w->stride_layer, w->stride_seq, w->stride_head} : SlotWeights{};
}

// The sequences of a call that has no tokens of its own.
cr_status check_slots(const cr_kv_layout* l, const cr_sequences* q) {
  if (l->n_layers < 1 || l->n_kv_heads < 1) return CR_ERR_DIMS;
  if (q->n_seqs < 1) return CR_ERR_OFFSETS;
  if (q->block_size < 1 || q->block_size > 1024 || (q->block_size & (q->block_size - 1)) ||
      q->max_blocks < 1)
    return CR_ERR_LAYOUT;
  if ((int64_t)q->max_blocks * q->block_size > kMostSlots) return CR_ERR_DIMS;
  // (a workgroup of up to 1024 threads for each layer, sequence and head)
  const int64_t ls = (int64_t)l->n_layers * q->n_seqs;
  if (ls > ((int64_t)1 << 32) / 1024 || !fits_launch(ls * l->n_kv_heads, 1024)) return CR_ERR_DIMS;
  return CR_OK;
}

cr_status check_weigh(const cr_kv_layout* l, const cr_sequences* q, int n_heads, Batch* b) {
  return check_attend(l, q, n_heads, 0, b);
}
// Which kernel a call takes, and its workspace.  Rows of a sequence and KV head:
//  - up to 16, what an instruction takes at once: a wave for each tile of keys (64
//    sequences of 8,192 slots, 32 query and 8 KV heads of 128: 227 us; four waves to a
//    tile's rows, three of them idle, 650);
//  - up to 512, where the table has room for at most 768 tiles: four waves share a
//    tile's rows (one sequence of 4,000 slots, the same heads: 9 us for 20 rows, 11 for
//    128, 19 for 512, 32 for 1,024; through LDS 16, 18, 24, 32);
//  - else the rows go through LDS for twice the keys (8,000 slots: 14, 17, 28, 41 us;
//    without 19, 20, 34, 55), and where tiles are few, units share a tile's rows (4,000
//    slots, 2,048 rows: 48 us; not shared 58).
struct WeighPlan {
  int kind = kWeighToken, slots = 0;
  uint64_t table = 0, info = 0, partial = 0, total = 0;
};
WeighPlan weigh_plan(const cr_kv_layout* l, const cr_sequences* q, const Batch& b, int n_heads) {
  WeighPlan p;
  if (!b.n_tokens) return p;
  const int group = n_heads / l->n_kv_heads;
  const int keys = weigh_keys((int)esize(l->dtype), l->head_dim);
  const int64_t slots = (int64_t)q->max_blocks * q->block_size;
  const auto tiles = [&](int n) { return (int64_t)q->n_seqs * ceil_div(slots, n) * l->n_kv_heads; };
  p.kind = b.most * group <= 16                                ? kWeighToken
           : b.most * group <= 512 && tiles(keys) <= kWeighSlots ? kWeighRows
                                                                 : kWeighWide;
  Arena a;
  if (b.off && q->n_seqs > kTableSeqs) p.table = a.take(((uint64_t)q->n_seqs + 1) * 4);
  if (p.kind == kWeighWide) {
    p.info = a.take(((uint64_t)b.n_tokens * n_heads + 64) * 32);
    if (tiles(2 * keys) * 2 <= kWeighSlots) {
      p.slots = kWeighSlots;
      p.partial = a.take((uint64_t)kWeighSlots * 2 * keys * 4);
    }
  }
  p.total = a.off;
  return p;
}

}  // namespace

extern "C" {

cr_status cr_weigh_workspace_bytes(const cr_kv_layout* layout, const cr_sequences* seqs,
                                   int32_t n_heads, uint64_t* bytes) {
  if (!layout || !seqs || !bytes) return CR_ERR_NULL;
  Batch b;
  const cr_status st = check_weigh(layout, seqs, n_heads, &b);
  if (st != CR_OK) return st;
  *bytes = weigh_plan(layout, seqs, b, n_heads).total;
  return CR_OK;
}

cr_status cr_weigh_keys(const void* kv, const cr_kv_layout* layout, int32_t layer,
                        const cr_sequences* seqs, const cr_rows* q, int32_t n_heads,
                        const cr_attend_options* options, const cr_key_weights* weights,
                        void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!kv || !layout || !seqs || !q || !options || !weights || !seqs->kv_lens || !seqs->block_table)
    return CR_ERR_NULL;
  const cr_attend_options& o = *options;
  Batch b;
  cr_status st = check_attend(layout, seqs, n_heads, o.shared_len, &b);
  if (st != CR_OK) return st;
  if (layer < 0 || layer >= layout->n_layers) return CR_ERR_DIMS;
  if ((st = check_scores(o, n_heads)) != CR_OK) return st;
  if ((st = check_blocks(layout, seqs)) != CR_OK) return st;
  if (!aligned(kv, 16)) return CR_ERR_LAYOUT;
  if ((st = check_rows(q, b.n_tokens, n_heads, layout->head_dim, false)) != CR_OK) return st;
  if ((st = check_weights(weights, layout->n_layers, layout->n_kv_heads, seqs)) != CR_OK) return st;
  if (b.n_tokens == 0) return CR_OK;
  if (!o.lse) return CR_ERR_NULL;
  const WeighPlan p = weigh_plan(layout, seqs, b, n_heads);
  if (p.total) {
    if (!workspace) return CR_ERR_NULL;
    if (workspace_bytes < p.total || !aligned(workspace, ALIGN)) return CR_ERR_WORKSPACE;
  }
  st = check_device();
  if (st != CR_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  WeighArgs a{};
  a.seqs = paged(layout, seqs);
  a.k = component(kv, layout, layer, 0);
  a.q = q->data;
  a.q_token = q->stride_token;
  a.q_head = q->stride_head;
  a.lse = o.lse;
  a.weights = slot_weights(weights);
  a.weights.data += (int64_t)layer * weights->stride_layer;
  a.n_tokens = (int)b.n_tokens;
  a.n_kv = layout->n_kv_heads;
  a.group = n_heads / layout->n_kv_heads;
  a.head_dim = layout->head_dim;
  a.lo = o.lo;
  a.hi = o.hi;
  set_scores(a, o, n_heads);
  char* ws = static_cast<char*>(workspace);
  a.kind = p.kind;
  a.slots = p.slots;
  // (a round of rows spans 64 queries of one head each, or fewer of up to 64 heads)
  a.near = q->stride_token < (1 << 23) && q->stride_head < (1 << 20) &&
           (64 * (q->stride_token + q->stride_head) + 256) * 4 < (int64_t)1 << 31;
  a.info = reinterpret_cast<RowInfo*>(ws + p.info);
  a.partial = reinterpret_cast<float*>(ws + p.partial);
  WeighTable tab{};
  a.ragged = b.off != nullptr;
  if (!a.ragged) {
    a.q_per_seq = (int)b.most;
  } else if (seqs->n_seqs <= kTableSeqs) {
    std::copy(b.off, b.off + seqs->n_seqs + 1, tab.q);
  } else {
    int* dev = reinterpret_cast<int*>(ws + p.table);
    CR_TRY(timed("weigh_table", s, [&] { return copy_table(b.off, seqs->n_seqs + 1, dev, s); }));
    a.q_off = dev;
  }
  CR_TRY(timed("weigh_keys", s, [&] {
    return layout->dtype == CR_DTYPE_BF16 ? weigh<bf16>(a, tab, s) : weigh<float>(a, tab, s); }));
  return CR_OK;
}

cr_status cr_choose_slots(const cr_kv_layout* layout, const cr_sequences* seqs,
                          const cr_key_weights* weights, const cr_choice* choice,
                          int32_t* kept, int32_t* kept_lens, void* stream) {
  if (!layout || !seqs || !weights || !choice || !kept || !kept_lens || !seqs->kv_lens)
    return CR_ERR_NULL;
  cr_status st = check_slots(layout, seqs);
  if (st != CR_OK) return st;
  if (choice->budget < 1 || choice->budget > kMostSlots || choice->first < 0 || choice->recent < 0)
    return CR_ERR_DIMS;
  // (a workgroup would read what another has written)
  if (lens_overlap(kept_lens, seqs->kv_lens, seqs->n_seqs) ||
      lens_overlap(kept_lens, choice->budgets, seqs->n_seqs))
    return CR_ERR_LAYOUT;
  if ((st = check_weights(weights, layout->n_layers, layout->n_kv_heads, seqs)) != CR_OK) return st;
  if ((st = check_device()) != CR_OK) return st;
  ChooseArgs a{};
  a.weights = slot_weights(weights);
  a.n_layers = layout->n_layers;
  a.n_seqs = seqs->n_seqs;
  a.n_kv = layout->n_kv_heads;
  a.max_len = seqs->max_blocks * seqs->block_size;
  a.lens = seqs->kv_lens;
  a.budgets = choice->budgets;
  a.budget = choice->budget;
  a.first = choice->first;
  a.recent = choice->recent;
  a.kept = kept;
  a.kept_lens = kept_lens;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  CR_TRY(timed("choose_slots", s, [&] { return choose(a, s); }));
  return CR_OK;
}

cr_status cr_compact_kv(void* kv, const cr_kv_layout* layout, const cr_sequences* seqs,
                        const int32_t* kept, int32_t budget, const int32_t* kept_lens,
                        const int32_t* table_out, int32_t max_blocks_out,
                        const cr_key_weights* weights, void* stream) {
  if (!kv || !layout || !seqs || !kept || !kept_lens || !seqs->kv_lens || !seqs->block_table)
    return CR_ERR_NULL;
  cr_status st = check_cache(layout);
  if (st != CR_OK) return st;
  if ((st = check_slots(layout, seqs)) != CR_OK) return st;
  if (budget < 1 || budget > kMostSlots) return CR_ERR_DIMS;
  // (with the lengths after for those before, every slot behind them would be dropped)
  if (lens_overlap(kept_lens, seqs->kv_lens, seqs->n_seqs)) return CR_ERR_LAYOUT;
  if (table_out && (max_blocks_out < 1 || (int64_t)max_blocks_out * seqs->block_size > kMostSlots))
    return CR_ERR_LAYOUT;
  if ((st = check_blocks(layout, seqs)) != CR_OK) return st;
  if (!aligned(kv, 16)) return CR_ERR_LAYOUT;
  if (weights &&
      (st = check_weights(weights, layout->n_layers, layout->n_kv_heads, seqs)) != CR_OK)
    return st;
  if ((st = check_device()) != CR_OK) return st;
  CompactArgs a{};
  a.seqs = paged(layout, seqs);
  a.kv = static_cast<char*>(kv);
  a.layer = layout->stride_layer;
  a.kv_step = layout->stride_kv;
  a.n_layers = layout->n_layers;
  a.n_kv = layout->n_kv_heads;
  a.element_bytes = (int)esize(layout->dtype);
  a.row_bytes = layout->head_dim * a.element_bytes;
  a.kept = kept;
  a.kept_lens = kept_lens;
  a.budget = budget;
  a.table_out = table_out;
  a.max_blocks_out = table_out ? max_blocks_out : seqs->max_blocks;
  a.weights = slot_weights(weights);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  CR_TRY(timed("compact_kv", s, [&] { return compact(a, s); }));
  return CR_OK;
}

cr_status cr_sample(const cr_logits* logits, const cr_sampling* options, const float* u,
                    int32_t* tokens, float* log_probs, void* stream) {
  if (!logits) return CR_ERR_NULL;
  if (logits->dtype != CR_DTYPE_BF16 && logits->dtype != CR_DTYPE_F32) return CR_ERR_DTYPE;
  if (logits->n_rows < 0 || !fits_launch(logits->n_rows, 1024) || logits->vocab < 1 ||
      logits->vocab > kMostVocab)
    return CR_ERR_DIMS;
  int64_t reach;
  if (logits->stride_row < 0 ||
      __builtin_mul_overflow(logits->stride_row, (int64_t)logits->n_rows, &reach) ||
      reach >= (int64_t)1 << 60 || !aligned(logits->data, esize(logits->dtype)))
    return CR_ERR_LAYOUT;
  if (logits->n_rows == 0) return CR_OK;
  if (!logits->data || !u || !tokens) return CR_ERR_NULL;
  const cr_status st = check_device();
  if (st != CR_OK) return st;
  SampleArgs a{};
  a.logits = logits->data;
  a.stride = logits->stride_row;
  a.n_rows = logits->n_rows;
  a.vocab = logits->vocab;
  a.temperature = 1.f;
  a.top_p = 1.f;
  if (options) {
    a.temperature = options->temperature;
    a.top_p = options->top_p;
    a.min_p = options->min_p;
    a.top_k = options->top_k;
    a.temperatures = options->temperatures;
    a.top_ps = options->top_ps;
    a.min_ps = options->min_ps;
    a.top_ks = options->top_ks;
  }
  a.u = u;
  a.tokens = tokens;
  a.log_probs = log_probs;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  CR_TRY(timed("sample", s, [&] {
    return logits->dtype == CR_DTYPE_BF16 ? sample<bf16>(a, s) : sample<float>(a, s); }));
  return CR_OK;
}

}  // extern "C"
