// Launchers of the kernels that keep an answer going (internal to the library):
// the weight of every cached slot, the choice of the slots that stay, their
// compaction, and sampling.
#pragma once
#include "serve.h"

namespace cr {

// Weights [layer][sequence][KV head][slot], fp32; strides in elements.
struct SlotWeights {
  float* data;
  int64_t layer, seq, head;
};

// ---- weights of one layer's slots.  weights.data is the layer's part.
struct WeighArgs {
  PagedSeqs seqs;
  const void *k, *q;
  const float* lse;                 // [n_tokens][n_heads]
  SlotWeights weights;
  int64_t q_token, q_head;
  int n_tokens, n_kv, group, head_dim;
  // where the sequences' queries begin: q_per_seq for each (ragged 0), or a
  // table, in device memory or (null) in the launch's WeighTable
  int ragged, q_per_seq;
  const int* q_off;
  const int *lo, *hi;               // device interval of every query, or null
  float scale_log2;                 // as in AttendArgs
  float cap_log2, scale_over_cap;
  int bias;
  float slopes_log2[kMaxQueryHeads];
  int kind;                         // kWeighToken, kWeighRows, kWeighWide
  // kWeighWide: what each row brings, [n_kv][n_tokens * group] and a chunk more; where
  // the tiles may be few, partial sums of `slots` units (else 0: no parts)
  struct RowInfo* info;
  float* partial;
  int slots;
  int near;                         // the rows of a round of transfers lie within 2^31 bytes
};
enum { kWeighToken = 0, kWeighRows = 1, kWeighWide = 2 };
constexpr int kWeighSlots = 768;
struct WeighTable {
  int q[kTableSeqs + 1];
};
// Keys of a wave's tile: what fits 64 registers (fp32: 32 at most).
constexpr int weigh_keys(int element_bytes, int head_dim) {
  const int row = element_bytes * head_dim;
  return row <= 256 && element_bytes == 2 ? 64 : row <= 512 ? 32 : 16;
}
constexpr int weigh_token_keys(int element_bytes, int head_dim) {
  return weigh_keys(element_bytes, head_dim) > 32 ? 32 : weigh_keys(element_bytes, head_dim);
}
// Tiles that the table has room for.
inline int64_t weigh_tiles(const WeighArgs& a, int keys) {
  return (int64_t)a.seqs.n_seqs * ((a.seqs.max_len + keys - 1) / keys);
}
template <typename T>
hipError_t weigh(const WeighArgs& a, const WeighTable& tab, hipStream_t s);

// ---- the slots that stay, of every layer, sequence and KV head.
struct ChooseArgs {
  SlotWeights weights;
  int n_layers, n_seqs, n_kv, max_len;
  const int *lens, *budgets;        // budgets null: budget for each
  int budget, first, recent;
  int *kept, *kept_lens;            // kept [layer][seq][head][budget]
};
hipError_t choose(const ChooseArgs& a, hipStream_t s);

// ---- the slots that stay moved to the front.
struct CompactArgs {
  PagedSeqs seqs;
  char* kv;
  int64_t layer, kv_step;           // strides in elements, as PagedSeqs
  int n_layers, n_kv, row_bytes, element_bytes;
  const int *kept, *kept_lens;
  int budget;
  const int* table_out;             // null: in place
  int max_blocks_out;
  SlotWeights weights;              // data null: none
};
hipError_t compact(const CompactArgs& a, hipStream_t s);

// ---- a token for every row of logits.
constexpr int kMostVocab = 1 << 19;
struct SampleArgs {
  const void* logits;
  int64_t stride;
  int n_rows, vocab;
  float temperature, top_p, min_p;
  int top_k;
  const float *temperatures, *top_ps, *min_ps;   // per row, or null
  const int* top_ks;
  const float* u;
  int* tokens;
  float* log_probs;                 // null: none
};
template <typename T>
hipError_t sample(const SampleArgs& a, hipStream_t s);

}  // namespace cr
