// Launchers of the kernels that answer over a paged cache (internal to the
// library): appending rotated keys and values, and attention over the pages.
#pragma once
#include <stdint.h>

#include "launch.h"

namespace cr {

constexpr int kMaxQueryHeads = 256;

// HIP launches fewer than 2^32 threads along a dimension.
constexpr bool fits_launch(int64_t workgroups, int threads) {
  return workgroups <= (((int64_t)1 << 32) - 1) / threads;
}

// One layer of a paged cache and the sequences in it.  Token t of sequence s
// lies in block table[s * max_blocks + (t >> shift)], row t & (2^shift - 1).
// lens and table are device memory that only the kernels read: a length below 0
// counts as 0, no slot from max_len on exists, and a block outside [0, n_blocks)
// is no block.
struct PagedSeqs {
  int64_t token, head, block;       // strides in elements
  int shift, n_blocks, max_blocks, max_len, n_seqs;
  const int *table, *lens;
};

// ---- append: K (rotated) and V of the new tokens into their pages, and the
// rotated queries.  New token i of sequence s has slot lens[s] - q_s + i.
struct AppendArgs {
  PagedSeqs seqs;
  void *k_cache, *v_cache;          // this layer's keys and values
  const void *k, *v, *q;            // q null: no queries
  void* q_out;
  int64_t k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
  int n_tokens, n_kv, n_heads, head_dim;
  const int* positions;             // device, null: the slot
  int rotate;                       // 0: copied as they are
};
// Heads (keys and queries) that a thread rotates: one while that leaves a CU one
// workgroup at most, else four that share their angles (one / two / four / eight
// heads: 64 tokens of 18 heads 5.7 / 6.3 / 6.8 / 10.0 us, 11,243 of 40 77 / 63 /
// 57 / 55); and the workgroups of 256 threads of a launch.
constexpr int append_heads(int64_t tokens, int64_t heads, int64_t head_dim) {
  return tokens * heads * (head_dim / 16) <= 256 * 256 ? 1 : 4;
}
constexpr int64_t append_groups(int64_t tokens, int64_t n_kv, int64_t heads, int64_t head_dim) {
  const int hpt = append_heads(tokens, heads, head_dim);
  const int64_t rotated = (heads + hpt - 1) / hpt * (head_dim / 16), copied = n_kv * (head_dim / 8);
  return (tokens * (rotated > copied ? rotated : copied) + 255) / 256;
}
template <typename T>
hipError_t append_kv(const AppendArgs& a, const KeyRope& kr, const int32_t* offsets,
                     hipStream_t s);

// ---- attention.  A unit is a tile of `rows` (query, head of the group) rows
// of one sequence and one KV head; see attend_kernel.h.
struct AttendArgs {
  PagedSeqs seqs;
  const void *k, *v;                // this layer's keys and values
  const void* q;
  int64_t q_token, q_head, o_token, o_head;
  void* o;
  float* lse;                       // [n_tokens][n_heads] or null
  int n_tokens, n_kv, group, head_dim;
  // where the sequences' queries and units begin: q_per_seq queries and
  // units_per_seq units for each (ragged 0), or a table, in device memory or
  // (null) in the launch's SeqTable
  int ragged, q_per_seq, units_per_seq, n_units, rows;
  const int *q_off, *unit_off;
  const int *lo, *hi;               // device interval of every query, or null
  float scale_log2;                 // score scale * log2(e)
  float cap_log2, scale_over_cap;   // cap * log2(e) (0: no cap), scale / cap
  int bias;                         // slopes are used
  float slopes_log2[kMaxQueryHeads];
  // keys of this pass: [key_begin, ...) of every sequence, or, with shared > 0,
  // [0, shared) of sequence 0's pages for the rows of all sequences
  int key_begin, shared;
  // splits of the keys: planned on the device from the lengths (slots > 0:
  // about that many items per KV head, at least min_tiles 64-key tiles each; no
  // more than slots items where there are at most one_round units; no split if
  // the longest unit takes at most chunk * split_cost + join_cost tiles, given
  // split_cost > 0), or fixed (shared: `splits` of split_tiles tiles), or none
  int slots, min_tiles, one_round, splits, split_tiles;
  float split_cost, join_cost;
  int always_partial;               // write partial results for the merge
  int2* unit_items;                 // [unit] first item and parts, for the merge
  float* part_o;                    // [item][kv head][rows][head_dim]
  float2* part_ml;                  // [item][kv head][rows] (max, sum)
};
// Rows of a wide unit: 128, or 64 where 128 rows' accumulators would leave a
// SIMD one wave (bf16 heads of 256: 327 / 241 us with 128 / 64 rows for 11 x 400
// tokens over 5,000 keys, 64 / 53 for 8 x 32; fp32 heads of 128: 50 / 36 for 60 x
// 3 over 300); and how many such workgroups a CU holds (fp32 heads over 192 take
// more than 256 registers even so).
constexpr int attend_rows(int element_bytes, int head_dim) {
  return head_dim > (element_bytes == 4 ? 96 : 128) ? 64 : 128;
}
constexpr int attend_resident(int element_bytes, int head_dim) {
  return element_bytes == 4 && head_dim > 192 ? 1 : 2;
}
// Offsets of a ragged batch of at most kTableSeqs sequences, passed by value:
// a launch less than a table in device memory (5 sequences: 4 us).
constexpr int kTableSeqs = 128;
struct SeqTable {
  int q[kTableSeqs + 1], unit[kTableSeqs + 1];
};
// Workgroups of a pass, one for each item and KV head, and their threads: two
// waves for 16 rows, else four.
constexpr int64_t attend_groups(int64_t items, int64_t n_kv) { return items * n_kv; }
constexpr int attend_threads(int rows) { return rows == 16 ? 128 : 256; }
template <typename T>
hipError_t attend(const AttendArgs& a, const SeqTable& tab, hipStream_t s);

// The partial results of the pass over the shared keys (splits 0: none).
struct SharedParts {
  int splits, rows;
  const float* part_o;
  const float2* part_ml;
};
// Rows that a workgroup (of 256 threads) of the merge joins, of at most `rows`
// rows in each of `tiles` units and KV heads: one while there are few (their parts
// are many), else as many as leave a row's dims a thread each (8 rather than 4
// rows: 13.7 rather than 21.5 us for 8 questions' 50,000 rows, 6.1 rather than 8.5
// for 12,000).  Few: 2,800 rows of 6 parts took 11.0 us one by one and 7.1 by
// eights, 1,024 rows of 18 parts 9.9 and 14.4
constexpr int merge_rows(int64_t tiles, int rows, int head_dim) {
  return tiles * rows <= 1024 ? 1 : head_dim <= 128 ? 8 : 4;
}
constexpr int64_t merge_groups(int64_t tiles, int rows, int head_dim) {
  const int per = merge_rows(tiles, rows, head_dim);
  return tiles * ((rows + per - 1) / per);
}
// Joins the partial results of a planned pass and those of the shared keys.  most_rows: rows of the longest sequence.
template <typename T>
hipError_t attend_merge(const AttendArgs& a, const SharedParts& pre, const SeqTable& tab,
                        int most_rows, hipStream_t s);

}  // namespace cr
