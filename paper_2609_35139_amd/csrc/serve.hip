// C ABI of answering over a paged cache: validation, the split of the work and
// the kernel sequence of cr_append_kv and cr_attend.  See include/cacherepair.h.
#include "../../include/cacherepair.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "profile.h"
#include "rules.h"
#include "serve.h"
#include "validate.h"

namespace {

using namespace cr;   // the helpers of validate.h and profile.h

constexpr int64_t kMostTokens = ((int64_t)1 << 31) - 256;

// The batch as the host sees it.
struct Batch {
  int64_t n_tokens = 0;
  int64_t most = 0;              // queries of the longest sequence
  const int32_t* off = nullptr;  // null: every sequence has n_tokens / n_seqs queries
};

cr_status check_cache(const cr_kv_layout* l) {
  if (l->n_layers < 1 || l->n_kv_heads < 1 || l->head_dim < 32 || l->head_dim > 256 ||
      l->head_dim % 32)
    return CR_ERR_DIMS;
  return check_dtype(l);
}

// The offsets and the table's extent (no device memory is read).
cr_status check_batch(const cr_sequences* q, Batch* b) {
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
cr_status check_rows(const cr_rows* r, int64_t n, int64_t heads, int64_t head_dim, bool written) {
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
cr_status check_blocks(const cr_kv_layout* l, const cr_sequences* q) {
  const cr_status st = check_page_strides(l, q->block_size, q->n_blocks, q->stride_block);
  if (st != CR_OK) return st;
  if (q->block_size > 1 && l->stride_token >= ((int64_t)1 << 32) / (int64_t)esize(l->dtype))
    return CR_ERR_LAYOUT;
  return CR_OK;
}

PagedSeqs paged(const cr_kv_layout* l, const cr_sequences* q) {
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
const char* component(const void* kv, const cr_kv_layout* l, int layer, int c) {
  return static_cast<const char*>(kv) +
         ((int64_t)layer * l->stride_layer + (int64_t)c * l->stride_kv) * (int64_t)esize(l->dtype);
}

// ------------------------------------------------------------- attention
// How one cr_attend call is cut up; a function of what the host knows, so the
// workspace can be sized ahead of the lengths.
struct Plan {
  int rows = 0, pre_rows = 0;    // rows of a unit of either pass
  int64_t units = 0;             // of the pass over each sequence's own keys
  int slots = 0, min_tiles = 0;  // its split (slots 0: none)
  float split_cost = 0.f, join_cost = 0.f;
  int64_t own_items = 0;         // partial results of that pass, per KV head
  int64_t pre_units = 0;         // units of the pass over the shared keys, its split
  int splits = 0, split_tiles = 0;
  uint64_t tables = 0, items = 0, own_ml = 0, own_o = 0, pre_ml = 0, pre_o = 0, total = 0;
};

// Whether one pass over the shared keys for the rows of all sequences takes less
// time than every sequence's own.  The pass and the merge of its parts add about
// 14 us to a call; it saves a unit's turn over the shared keys for each unit of
// the sequences.  What a unit takes per key and KV head, with the chip full
// (bf16, 128 dims, in picoseconds): 16 rows 26 (reading the keys, which lie in
// the caches by then), wide units 64, or 45 where rows are missing.  Measured
// with 32 query and 8 KV heads, shared pass against none, 100 keys more each: 32
// sequences of one token over 2048 shared keys 31 / 29 us, over 16384 46 / 121;
// of 8 tokens over 2048 51 / 45 us, over 16384 101 / 207; of 32 tokens, which
// fill their units, 322 / 289.  Other types and dims by the bytes of a narrow
// unit's keys and the matrix instructions of a wide one's: of one token, fp32 of
// 128 dims over 512 42 / 38, over 2048 47 / 80, bf16 of 64 over 2048 26.2 / 25.6,
// over 16384 36 / 81, of 256 over 2048 45 / 89; of 8 tokens, fp32 of 64 dims over
// 512 46.0 / 47.5 (it takes the slower), over 2048 77 / 110, bf16 of 256 over 512
// 50 / 36, over 16384 202 / 299.
bool shared_pays(const cr_kv_layout* l, const Batch& b, int G, const Plan& p, int shared) {
  const double elt = (double)esize(l->dtype), D = l->head_dim;
  const double wide = D / 128 * (elt == 4 ? 8 : 1) * attend_rows((int)elt, (int)D) / 128;
  const double own = p.rows == 16 ? 26 * D / 128 * elt / 2 : 45 * wide;
  const double pre = p.pre_rows == 16 ? 26 * D / 128 * elt / 2 : 64 * wide;
  const double per_key = own * (double)p.units - pre * (double)ceil_div(b.n_tokens * G, p.pre_rows);
  // (units that were not to be split would leave no partial results otherwise)
  const double join = p.slots ? 0 : 2.4 * (double)p.units * p.rows * D;
  return l->n_kv_heads * (per_key * shared - join) > 16e6;
}

Plan attend_plan(const cr_kv_layout* l, const cr_sequences* q, const Batch& b, int n_heads,
                 int shared) {
  Plan p;
  const int G = n_heads / l->n_kv_heads, D = l->head_dim, H = l->n_kv_heads;
  const int wide = attend_rows((int)esize(l->dtype), D);
  p.rows = b.most * G <= 16 ? 16 : wide;
  p.pre_rows = b.n_tokens * G <= 16 ? 16 : wide;
  auto tiles = [&](int64_t n) { return ceil_div(n * G, p.rows); };
  if (b.off) {
    for (int s = 0; s < q->n_seqs; ++s) p.units += tiles(b.off[s + 1] - b.off[s]);
  } else {
    p.units = q->n_seqs * tiles(b.most);
  }
  Arena a;
  if (b.off && q->n_seqs > kTableSeqs) p.tables = a.take(2 * ((uint64_t)q->n_seqs + 1) * 4);
  // split the keys unless the units fill the chip by themselves (single tokens
  // over 64 to 8,000 keys, 8 KV heads, split / whole: 128 sequences 176 / 202 us,
  // 256 342 / 356; 512 over up to 2,000 keys 283 / 234; wide units: 64 x 32 tokens
  // over 1,000 keys 74 / 65)
  int resident = 2;
  bool two_rounds = false;
  if (p.units * H < (p.rows == 16 ? 4096 : 512)) {
    // one round of the workgroups that a CU holds (two, but one where a wave
    // takes more than 256 registers: 52.6 / 45.9 us with parts for 512 / 256 of
    // those for 5 x 32 fp32 questions of 128 dims over 3,000 keys), or two rounds
    // where the units by themselves nearly fill one (their ragged lengths then
    // even out: 64 of the sequences above 94 / 101 us with / without)
    resident = p.rows == 16 ? 2 : attend_resident((int)esize(l->dtype), D);
    const int round = 256 * resident;
    p.slots = (int)std::max<int64_t>(1, round / H);
    // wide units that fill between half and two thirds of a round: three parts
    // each in two rounds, where a tile takes long next to the merge (11 x 400
    // tokens over 5,000 keys, 2 KV heads: bf16 of 256 dims 241 -> 207 us, fp32 of
    // 192 1289 -> 909; bf16 of 128 dims lost 5 to 20 us)
    if (p.rows != 16 && (D > 128 || l->dtype == CR_DTYPE_F32) && p.units * 2 > p.slots &&
        p.units * 3 <= p.slots * 2)
      p.slots *= 2;
    two_rounds = p.rows == 16 && p.units * 4 > p.slots * 3;
    if (two_rounds) p.slots = (int)std::max<int64_t>(1, 1024 / H);
    // a part has at least two tiles of 64 keys, or one for fp32, where a tile
    // takes eight times as long: 4 / 2 / 1 tiles took 39 / 28.9 / 24.4 us for 8 x
    // 161 fp32 questions over 769 keys, 42 / 38.4 / 38.5 us for bf16 documents,
    // and one took 44.0 instead of 40.4 us for 9 bf16 sequences over 1177 keys
    p.min_tiles = l->dtype == CR_DTYPE_F32 ? 1 : 2;
    // so few keys as the table can hold are not worth a merge: 128 KB of a head's
    // for single tokens (64 KB for fp32), 512 keys at most (split / whole: 400 keys
    // of 64 dims 13.5 / 9.6 us, 500 of 128 16.9 / 13.7, 400 of 256 16.8 / 20.4; fp32
    // of 128 dims 100 keys 13.5 / 13.5, 200 15.5 / 18.4)
    const int64_t row = D * (int64_t)esize(l->dtype), few = l->dtype == CR_DTYPE_F32 ? 1 << 16 : 1 << 17;
    if ((int64_t)q->max_blocks * q->block_size <=
        (p.rows == 16 ? std::min<int64_t>(512, few / row) : 128 * p.min_tiles))
      p.slots = 0;
  }
  if (shared_pays(l, b, G, p, shared)) {
    p.pre_units = ceil_div(b.n_tokens * G, p.pre_rows);
    const int64_t key_tiles = ceil_div(shared, 64);
    const int64_t want = std::max<int64_t>(1, 512 / (p.pre_units * H));
    p.split_tiles = (int)std::max<int64_t>(2, ceil_div(key_tiles, want));
    p.splits = (int)ceil_div(key_tiles, p.split_tiles);
  }
  // Nor single tokens of much the same lengths that fill the chip, or a unit of
  // up to two tiles more than a part (64 tokens, 8 KV heads, split / whole: 200
  // keys 29 / 24 us, 400 35 / 30, 1,000 57 / 53; 100 tokens over 4,000 378 / 304).
  if (p.slots && !p.pre_units && p.rows == 16 && l->dtype == CR_DTYPE_BF16) {
    p.split_cost = two_rounds ? std::max(1.f, 1.5f * (float)p.slots / (float)p.units) : 1.f;
    p.join_cost = 2.f;
  }
  // No split of wide units where it gains less than the merge takes: 2 us and 2.4 us for every
  // million sums, at 2 us for a wide bf16 tile of 128 dims.  A workgroup that
  // has its CU to itself takes two thirds of the time per tile (split_cost 1.5 / 1:
  // 16 sequences of 32 tokens over 300 keys 25.8 / 33.0 us, 24 over 600 36.3 /
  // 42.2, 8 to 24 over 1200 and more even), and with more
  // units than fit one round a split pays for very uneven lengths alone.  20
  // sequences of 32 tokens, 300 keys, 8 KV heads: 36 us split, 28 in one part;
  // 32 of them over 600 keys 48 and 37.5, over 2400 95 and 107; a prompt of 2000
  // tokens, 63 units, over 4800 keys 313 and 216.
  if (p.slots && !p.pre_units && p.rows != 16) {
    const double tile = 2.0 * D / 128 * p.rows / 128 * (l->dtype == CR_DTYPE_F32 ? 8 : 1);
    p.split_cost = p.units > p.slots * 3 / 4 ? 2.f : p.units * H <= 256 && resident > 1 ? 1.5f : 1.f;
    p.join_cost = (float)((2 + 2.4e-6 * (double)p.units * H * p.rows * D) / tile);
  }
  p.own_items = p.slots ? p.units + p.slots : p.pre_units ? p.units : 0;
  if (p.own_items) p.items = a.take((uint64_t)p.units * 8);
  const uint64_t own = (uint64_t)p.own_items * H * p.rows;
  const uint64_t pre = (uint64_t)p.pre_units * p.splits * H * p.pre_rows;
  p.own_ml = a.take(own * 8);
  p.own_o = a.take(own * D * 4);
  p.pre_ml = a.take(pre * 8);
  p.pre_o = a.take(pre * D * 4);
  p.total = a.off;
  return p;
}

// Whether every launch of a planned call is one that HIP makes.
bool launches_fit(const cr_kv_layout* l, const Batch& b, int n_heads, const Plan& p) {
  const int64_t H = l->n_kv_heads, G = n_heads / H;
  const int most_rows = (int)std::min<int64_t>(b.most * G, p.rows);
  return fits_launch(attend_groups(p.units + p.slots, H), attend_threads(p.rows)) &&
         fits_launch(attend_groups(p.pre_units * p.splits, H), attend_threads(p.pre_rows)) &&
         (!p.own_items || fits_launch(merge_groups(p.units * H, most_rows, l->head_dim), 256));
}

cr_status check_attend(const cr_kv_layout* l, const cr_sequences* q, int n_heads, int shared,
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

template <typename T>
cr_status attend_impl(const void* kv, const cr_kv_layout* l, int layer, const cr_sequences* q,
                      const Batch& b, const Plan& p, const cr_rows* qr, const cr_rows* out,
                      int n_heads, const cr_attend_options& o, char* ws, hipStream_t s) {
  AttendArgs a{};
  a.seqs = paged(l, q);
  a.k = component(kv, l, layer, 0);
  a.v = component(kv, l, layer, 1);
  a.q = qr->data;
  a.q_token = qr->stride_token;
  a.q_head = qr->stride_head;
  a.o = out->data;
  a.o_token = out->stride_token;
  a.o_head = out->stride_head;
  a.lse = o.lse;
  a.n_tokens = (int)b.n_tokens;
  a.n_kv = l->n_kv_heads;
  a.group = n_heads / l->n_kv_heads;
  a.head_dim = l->head_dim;
  a.rows = p.rows;
  a.n_units = (int)p.units;
  a.lo = o.lo;
  a.hi = o.hi;
  const double scale = o.scale > 0.f ? o.scale : 1.0 / std::sqrt((double)l->head_dim);
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
  SeqTable tab{};
  a.ragged = b.off != nullptr;
  if (!a.ragged) {
    a.q_per_seq = (int)b.most;
    a.units_per_seq = (int)ceil_div(b.most * a.group, p.rows);
  } else if (q->n_seqs <= kTableSeqs) {
    for (int i = 0; i <= q->n_seqs; ++i) {
      tab.q[i] = b.off[i];
      tab.unit[i] = i == 0 ? 0
                           : tab.unit[i - 1] +
                                 (int)ceil_div((int64_t)(b.off[i] - b.off[i - 1]) * a.group, p.rows);
    }
  } else {
    const int n = q->n_seqs + 1;
    int* dev = reinterpret_cast<int*>(ws + p.tables);
    CR_TRY(timed("attend_table", s, [&] {
      int32_t buf[512];
      int64_t unit = 0;
      for (int i0 = 0; i0 < 2 * n; i0 += 512) {
        const int m = std::min(512, 2 * n - i0);
        for (int i = i0; i < i0 + m; ++i) {
          if (i > n) unit += ceil_div((int64_t)(b.off[i - n] - b.off[i - n - 1]) * a.group, p.rows);
          buf[i - i0] = i < n ? b.off[i] : (int32_t)unit;
        }
        const hipError_t e = copy_table(buf, m, dev + i0, s);
        if (e != hipSuccess) return e;
      }
      return hipSuccess; }));
    a.q_off = dev;
    a.unit_off = dev + n;
  }
  a.slots = p.slots;
  a.min_tiles = p.min_tiles;
  a.split_cost = p.split_cost;
  a.join_cost = p.join_cost;
  a.one_round = p.slots * 3 / 4;
  a.unit_items = reinterpret_cast<int2*>(ws + p.items);
  a.part_ml = reinterpret_cast<float2*>(ws + p.own_ml);
  a.part_o = reinterpret_cast<float*>(ws + p.own_o);
  SharedParts parts{};
  if (p.pre_units) {
    AttendArgs pre = a;
    pre.shared = o.shared_len;
    pre.rows = p.pre_rows;
    pre.n_units = (int)p.pre_units;
    pre.slots = 0;
    pre.splits = p.splits;
    pre.split_tiles = p.split_tiles;
    pre.always_partial = 1;
    pre.part_ml = reinterpret_cast<float2*>(ws + p.pre_ml);
    pre.part_o = reinterpret_cast<float*>(ws + p.pre_o);
    parts = SharedParts{p.splits, p.pre_rows, pre.part_o, pre.part_ml};
    a.key_begin = o.shared_len;
    a.always_partial = 1;
    CR_TRY(timed("attend_shared", s, [&] { return attend<T>(pre, tab, s); }));
  }
  CR_TRY(timed("attend", s, [&] { return attend<T>(a, tab, s); }));
  if (p.own_items) {
    const int most_rows = (int)std::min<int64_t>(b.most * a.group, p.rows);
    CR_TRY(timed("attend_merge", s, [&] { return attend_merge<T>(a, parts, tab, most_rows, s); }));
  }
  return CR_OK;
}

}  // namespace

extern "C" {

cr_status cr_append_kv(void* kv, const cr_kv_layout* layout, int32_t layer,
                       const cr_sequences* seqs, const cr_rows* k, const cr_rows* v,
                       const cr_rows* q, const cr_rows* q_out, int32_t n_heads,
                       const cr_rope* rope, const int32_t* positions, void* stream) {
  if (!kv || !layout || !seqs || !k || !v || !seqs->kv_lens || !seqs->block_table)
    return CR_ERR_NULL;
  if (!q != !q_out) return CR_ERR_NULL;
  cr_status st = check_cache(layout);
  if (st != CR_OK) return st;
  Batch b;
  st = check_batch(seqs, &b);
  if (st != CR_OK) return st;
  if (layer < 0 || layer >= layout->n_layers) return CR_ERR_DIMS;
  if (q && (n_heads < 1 || n_heads > (1 << 16))) return CR_ERR_DIMS;
  if (layout->n_kv_heads > (1 << 16)) return CR_ERR_DIMS;
  st = check_blocks(layout, seqs);
  if (st != CR_OK) return st;
  if (!aligned(kv, 16)) return CR_ERR_LAYOUT;
  KeyRope kr{};
  kr.half = layout->head_dim / 2;
  if (rope) {
    st = key_rope_of(rope, layout->head_dim, &kr);
    if (st != CR_OK) return st;
  }
  const int64_t H = layout->n_kv_heads, D = layout->head_dim;
  if ((st = check_rows(k, b.n_tokens, H, D, false)) != CR_OK) return st;
  if ((st = check_rows(v, b.n_tokens, H, D, false)) != CR_OK) return st;
  if (q) {
    if ((st = check_rows(q, b.n_tokens, n_heads, D, false)) != CR_OK) return st;
    if ((st = check_rows(q_out, b.n_tokens, n_heads, D, true)) != CR_OK) return st;
    // in place only element on element
    if (q->data == q_out->data &&
        (q->stride_token != q_out->stride_token || q->stride_head != q_out->stride_head))
      return CR_ERR_LAYOUT;
  }
  // (in 64 bits: tokens below 2^31, heads at most 2^17)
  if (!fits_launch(append_groups(b.n_tokens, H, H + (q ? n_heads : 0), D), 256)) return CR_ERR_DIMS;
  if (b.n_tokens == 0) return CR_OK;
  st = check_device();
  if (st != CR_OK) return st;
  AppendArgs a{};
  a.seqs = paged(layout, seqs);
  a.k_cache = const_cast<char*>(component(kv, layout, layer, 0));
  a.v_cache = const_cast<char*>(component(kv, layout, layer, 1));
  a.k = k->data; a.k_token = k->stride_token; a.k_head = k->stride_head;
  a.v = v->data; a.v_token = v->stride_token; a.v_head = v->stride_head;
  if (q) {
    a.q = q->data; a.q_token = q->stride_token; a.q_head = q->stride_head;
    a.q_out = q_out->data; a.o_token = q_out->stride_token; a.o_head = q_out->stride_head;
    a.n_heads = n_heads;
  }
  a.n_tokens = (int)b.n_tokens;
  a.n_kv = layout->n_kv_heads;
  a.head_dim = layout->head_dim;
  a.positions = positions;
  a.rotate = rope != nullptr;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  CR_TRY(timed("append_kv", s, [&] {
    return layout->dtype == CR_DTYPE_BF16 ? append_kv<bf16>(a, kr, b.off, s)
                                          : append_kv<float>(a, kr, b.off, s); }));
  return CR_OK;
}

cr_status cr_attend_workspace_bytes(const cr_kv_layout* layout, const cr_sequences* seqs,
                                    int32_t n_heads, int32_t shared_len, uint64_t* bytes) {
  if (!layout || !seqs || !bytes) return CR_ERR_NULL;
  Batch b;
  const cr_status st = check_attend(layout, seqs, n_heads, shared_len, &b);
  if (st != CR_OK) return st;
  const Plan p = b.n_tokens ? attend_plan(layout, seqs, b, n_heads, shared_len) : Plan{};
  if (b.n_tokens && !launches_fit(layout, b, n_heads, p)) return CR_ERR_DIMS;
  *bytes = p.total;
  return CR_OK;
}

cr_status cr_attend(const void* kv, const cr_kv_layout* layout, int32_t layer,
                    const cr_sequences* seqs, const cr_rows* q, const cr_rows* out,
                    int32_t n_heads, const cr_attend_options* options, void* workspace,
                    uint64_t workspace_bytes, void* stream) {
  if (!kv || !layout || !seqs || !q || !out || !seqs->kv_lens || !seqs->block_table)
    return CR_ERR_NULL;
  const cr_attend_options o = options ? *options : cr_attend_options{};
  Batch b;
  cr_status st = check_attend(layout, seqs, n_heads, o.shared_len, &b);
  if (st != CR_OK) return st;
  if (layer < 0 || layer >= layout->n_layers) return CR_ERR_DIMS;
  if (!(o.scale >= 0.f) || !std::isfinite(o.scale) || !(o.softcap >= 0.f) ||
      !std::isfinite(o.softcap))
    return CR_ERR_DIMS;
  for (int h = 0; o.slopes && h < n_heads; ++h)
    if (!std::isfinite(o.slopes[h])) return CR_ERR_DIMS;
  st = check_blocks(layout, seqs);
  if (st != CR_OK) return st;
  if (!aligned(kv, 16)) return CR_ERR_LAYOUT;
  const int64_t D = layout->head_dim;
  if ((st = check_rows(q, b.n_tokens, n_heads, D, false)) != CR_OK) return st;
  if ((st = check_rows(out, b.n_tokens, n_heads, D, true)) != CR_OK) return st;
  if (q->data == out->data) return CR_ERR_LAYOUT;
  if (b.n_tokens == 0) return CR_OK;
  const Plan p = attend_plan(layout, seqs, b, n_heads, o.shared_len);
  if (!launches_fit(layout, b, n_heads, p)) return CR_ERR_DIMS;
  if (p.total) {
    if (!workspace) return CR_ERR_NULL;
    if (workspace_bytes < p.total || !aligned(workspace, ALIGN)) return CR_ERR_WORKSPACE;
  }
  st = check_device();
  if (st != CR_OK) return st;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  return layout->dtype == CR_DTYPE_BF16
             ? attend_impl<bf16>(kv, layout, layer, seqs, b, p, q, out, n_heads, o, ws, s)
             : attend_impl<float>(kv, layout, layer, seqs, b, p, q, out, n_heads, o, ws, s);
}

}  // extern "C"
