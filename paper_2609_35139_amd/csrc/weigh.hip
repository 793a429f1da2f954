// How much attention every cached slot receives (gfx950 MFMA):
//   W[s, h, j] += sum over the queries t of sequence s and the heads g of KV
//   head h's group of exp(x(t, g, j) - lse[t, g]),
// x the score of cr_attend (scaled, capped, biased) and lse the logarithm of
// its row's sum that cr_attend leaves, over the keys that t sees.
//
// Nothing is joined between keys, so a wave keeps a tile of keys in registers
// and walks the rows (query, head of the group) that see it.  Scores are formed
// transposed, S^T = K Q^T, in 16x16 atoms: a lane holds four consecutive keys of
// one row, so the row's lse and interval are a register each, the sum over the
// rows is register work, and the 16 lanes that share keys add up once, at the
// tile's end.  A lane's partial sums leave the exchange with one key each, so
// the weights are read and written in whole lines, and no order of the sum
// depends on anything but the sizes.
#include <climits>

#include "answer.h"
#include "scores.h"

namespace cr {

// Queries of a sequence: first token and number.
struct Queries { int tok0, nq; };
__device__ __forceinline__ Queries queries_of(const WeighArgs& a, const WeighTable& tab, int s) {
  if (!a.ragged) return {s * a.q_per_seq, a.q_per_seq};
  const int o = a.q_off ? a.q_off[s] : tab.q[s], e = a.q_off ? a.q_off[s + 1] : tab.q[s + 1];
  return {o, e - o};
}
// Tiles of KT keys of a sequence that has queries.
template <int KT>
__device__ __forceinline__ int key_tiles(const WeighArgs& a, const WeighTable& tab, int s) {
  if (queries_of(a, tab, s).nq == 0) return 0;
  return (min(seq_len(a.seqs, s), a.seqs.max_len) + KT - 1) / KT;
}

// Sums v[0..N) over the 16 lanes of a row of lanes (c16): lane c16 is left with
// the total of element c16 % N.  In a fixed order.
template <int N>
__device__ __forceinline__ float sum_to_lane(float (&v)[N], int c16) {
  int n = N;
#pragma unroll
  for (int b = 1; b < 16; b <<= 1) {
    if (n > 1) {
      n >>= 1;
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        if (j >= n) continue;
        const bool odd = (c16 & b) != 0;
        const float keep = odd ? v[2 * j + 1] : v[2 * j], send = odd ? v[2 * j] : v[2 * j + 1];
        v[j] = keep + __shfl_xor(send, b);
      }
    } else {
      v[0] += __shfl_xor(v[0], b);
    }
  }
  return v[0];
}

// Tile t of all sequences' tiles, in order: its sequence and the tile within it.  The
// same in every wave; the first 64 sequences' tiles stay in a register.
template <int KT>
struct Tiles {
  const WeighArgs& a;
  const WeighTable& tab;
  int lane, first64;
  long long total;
  __device__ __forceinline__ Tiles(const WeighArgs& a, const WeighTable& tab)
      : a(a), tab(tab), lane(threadIdx.x & 63) {
    first64 = lane < a.seqs.n_seqs ? key_tiles<KT>(a, tab, lane) : 0;
    total = 0;
    for (int s0 = 0; s0 < a.seqs.n_seqs; s0 += 64) {
      long long t = at(s0);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
      total += t;
    }
  }
  __device__ __forceinline__ int at(int s0) const {
    return s0 == 0 ? first64 : s0 + lane < a.seqs.n_seqs ? key_tiles<KT>(a, tab, s0 + lane) : 0;
  }
  __device__ __forceinline__ int2 find(long long t) const {
    long long base = 0;
    for (int s0 = 0; s0 < a.seqs.n_seqs; s0 += 64) {
      const int mine = at(s0);
      long long incl = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const long long x = __shfl_up(incl, o);
        if (lane >= o) incl += x;
      }
      const unsigned long long hit = __ballot(mine > 0 && base + incl > t);
      if (hit) {
        const int l = __ffsll(hit) - 1;
        const long long before = base + __shfl(incl, l) - __shfl(mine, l);
        return make_int2(__builtin_amdgcn_readfirstlane(s0 + l),
                         __builtin_amdgcn_readfirstlane((int)(t - before)));
      }
      base += __shfl(incl, 63);
    }
    return make_int2(-1, 0);
  }
};

// A wave's tile of keys [k0, k0 + KT) below n: fragments, and of each atom a bit for
// every key that lies in no block.
template <typename T, int D, int KT>
struct KeyTile {
  using MM = Mma16<T>;
  using frag = typename MM::frag;
  static constexpr int KA = KT / 16, QF = D / MM::KSTEP;
  frag kf[KA][QF];
  unsigned none[KA];
  __device__ __forceinline__ void load(const WeighArgs& a, int s, int head, int k0, int n) {
    const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int shift = a.seqs.shift, page_mask = (1 << shift) - 1;
    const int* table = a.seqs.table + (int64_t)s * a.seqs.max_blocks;
    const T* kbase = static_cast<const T*>(a.k) + (int64_t)head * a.seqs.head + g * MM::KPL;
#pragma unroll
    for (int x = 0; x < KA; ++x) {
      const int key = min(k0 + x * 16 + c16, n - 1);
      const int id = table[key >> shift];
      const bool ok = id >= 0 && id < a.seqs.n_blocks;
      none[x] = (unsigned)__ballot(!ok) & 0xffffu;
      const T* p = kbase + (ok ? (int64_t)id * a.seqs.block : 0) +
                   (int64_t)(key & page_mask) * a.seqs.token;
#pragma unroll
      for (int kk = 0; kk < QF; ++kk) kf[x][kk] = load_frag<T, frag>(p + kk * MM::KSTEP);
    }
  }
  __device__ __forceinline__ bool bad() const {
    unsigned b = 0;
#pragma unroll
    for (int x = 0; x < KA; ++x) b |= none[x];
    return b != 0;
  }
};

// What a row (query, head of the group) brings: its interval of keys, lse in exp2 units
// as the sum of two numbers, the second as a factor (one rounding of a lse of 20 would
// put the whole row off by 2^-20), its slot and slope.
struct __align__(16) RowInfo {
  int lo, hi;
  float ref, factor;
  int p;
  float slope;
  int pad[2];
};
// Row r of a sequence's rows for KV head `head`; a row that saw nothing (lse -inf) sees
// nothing.
__device__ __forceinline__ RowInfo row_info(const WeighArgs& a, int len, const Queries& qs, int head,
                                            int i, int g) {
  const int64_t t = qs.tok0 + i;
  const int hd = head * a.group + g, most = min(len, a.seqs.max_len);
  RowInfo r;
  r.p = len - qs.nq + i;
  r.hi = max(min(a.hi ? a.hi[t] : r.p + 1, most), 0);
  r.lo = a.lo ? max(a.lo[t], 0) : 0;
  const float lse = a.lse[t * a.n_kv * a.group + hd];
  if (lse == -INFINITY) r.hi = r.lo = 0;
  r.ref = lse * kLog2e;
  const float rest = __builtin_fmaf(lse, kLog2e, -r.ref);
  r.factor = isfinite(rest) ? __builtin_amdgcn_exp2f(-rest) : 1.f;
  r.slope = a.bias ? a.slopes_log2[hd] : 0.f;
  return r;
}

// Adds the shares of 16 rows to a tile's sums: lane (g, c16) holds row c16 and keys 16 x
// + 4 g + [0, 4).  general: scores are capped or biased; whole: every row sees every key.
template <typename T, int D, int KT>
__device__ __forceinline__ void add_rows(const WeighArgs& a, bool general, const KeyTile<T, D, KT>& keys, int k0,
                                         const typename Mma16<T>::frag (&qf)[D / Mma16<T>::KSTEP],
                                         const RowInfo& row, bool whole, float (&sum)[KT / 4]) {
  using MM = Mma16<T>;
  constexpr int KA = KT / 16, QF = D / MM::KSTEP;
  f32x4 sc[KA];
#pragma unroll
  for (int x = 0; x < KA; ++x) {
    sc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < QF; ++kk) sc[x] = MM::mma(keys.kf[x][kk], qf[kk], sc[x]);
  }
  if (general) {
    const int first = row.p - k0 - 4 * (lane_again() >> 4);
#pragma unroll
    for (int x = 0; x < KA; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y = sc[x][e] * a.scale_log2;
        if (a.cap_log2 > 0.f) {
          const float u = sc[x][e] * a.scale_over_cap;
          y = fabsf(u) > kCapSmall ? a.cap_log2 * tanh_of<T>(u) : y * tanh_over(u);
        }
        sc[x][e] = y - row.slope * fabsf((float)(first - x * 16 - e)) - row.ref;
      }
  } else {
#pragma unroll
    for (int x = 0; x < KA; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[x][e] = __builtin_fmaf(sc[x][e], a.scale_log2, -row.ref);
  }
#pragma unroll
  for (int x = 0; x < KA; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[x][e] = __builtin_amdgcn_exp2f(sc[x][e]);
  if (!whole) {
    // (what depends on the lane is formed anew: kept from call to call it would fill the
    // registers of the code above)
    const int shift = 4 * (lane_again() >> 4), first = k0 + shift;
#pragma unroll
    for (int x = 0; x < KA; ++x) {
      const unsigned none = keys.none[x] >> shift;
      const int lo = row.lo - first - x * 16, hi = row.hi - first - x * 16;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sc[x][e] = ((e >= lo) & (e < hi) & !((none >> e) & 1)) ? sc[x][e] : 0.f;
    }
  }
#pragma unroll
  for (int x = 0; x < KA; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      sum[x * 4 + e] = __builtin_fmaf(sc[x][e], row.factor, sum[x * 4 + e]);
}

// ---- up to 16 rows in every sequence (single tokens): each wave has tiles of its own, a
// run of them, and keeps the rows while the sequence is the same.  Bound by the keys'
// bytes: 64 sequences of 73 to 15,144 slots (170,000 in all), 8 KV heads of 128: 82 us,
// 4.4 TB/s; tiles of 64 keys leave fewer waves to a CU (99 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void weigh_token_kernel(WeighArgs a, WeighTable tab) {
  using MM = Mma16<T>;
  using frag = typename MM::frag;
  constexpr int KPL = MM::KPL, KSTEP = MM::KSTEP, QF = D / KSTEP;
  constexpr int KT = weigh_token_keys(sizeof(T), D), KA = KT / 16;
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.n_kv;
  const int worker = blockIdx.x / a.n_kv * 4 + wave, workers = gridDim.x / a.n_kv * 4;
  const Tiles<KT> tiles(a, tab);
  const long long per = (tiles.total + workers - 1) / workers;
  long long t0 = worker * per;
  const long long t1 = min(tiles.total, t0 + per);
  if (t0 >= t1) return;
  const int2 at = tiles.find(t0);
  int s = at.x, tile = at.y, n = 0;
  if (s < 0) return;
  RowInfo row{};
  frag qf[QF];
  auto enter = [&] {                       // sequence s: its rows
    const int len = seq_len(a.seqs, s);
    n = min(len, a.seqs.max_len);
    const Queries qs = queries_of(a, tab, s);
    const int n_rows = qs.nq * a.group, r = min(c16, max(n_rows - 1, 0)), i = r / a.group;
    if (n_rows == 0) { n = 0; return; }
    row = row_info(a, len, qs, head, i, r - i * a.group);
    if (c16 >= n_rows) row.hi = row.lo = 0;
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(qs.tok0 + i) * a.q_token +
                  (int64_t)(head * a.group + r - i * a.group) * a.q_head;
#pragma unroll
    for (int kk = 0; kk < QF; ++kk) qf[kk] = load_frag<T, frag>(qp + kk * KSTEP + g * KPL);
  };
  enter();
  for (; t0 < t1; ++t0, ++tile) {
    while (tile * KT >= n) {               // the next sequence with a tile
      if (++s >= a.seqs.n_seqs) return;
      tile = 0;
      enter();
    }
    const int k0 = tile * KT;
    KeyTile<T, D, KT> keys;
    keys.load(a, s, head, k0, n);
    float sum[KA * 4];
#pragma unroll
    for (int x = 0; x < KA * 4; ++x) sum[x] = 0.f;
    const bool whole = !keys.bad() && __all(row.lo <= k0 && row.hi >= k0 + KT);
    add_rows<T, D, KT>(a, a.cap_log2 > 0.f || a.bias, keys, k0, qf, row, whole, sum);
    // one key per lane: atom x = id / 4, key 16 x + 4 g + id % 4, id = c16 % (4 KA)
    const float mine = sum_to_lane(sum, c16);
    const int id = c16 % (KA * 4), at = (id >> 2) * 16 + 4 * g + (id & 3);
    if (c16 < KA * 4 && k0 + at < n)
      a.weights.data[(int64_t)s * a.weights.seq + (int64_t)head * a.weights.head + k0 + at] += mine;
  }
}

// ---- some rows: the four waves of a workgroup share a tile's rows, read where they lie.
// Bound by latency: every wave waits for its 16 rows in turn, so this is for calls that
// a CU is done with in a few rounds (20 rows over 4,000 slots: 9 us).
template <typename T, int D>
__global__ __launch_bounds__(256) void weigh_rows_kernel(WeighArgs a, WeighTable tab) {
  using MM = Mma16<T>;
  using frag = typename MM::frag;
  constexpr int KPL = MM::KPL, KSTEP = MM::KSTEP, QF = D / KSTEP;
  constexpr int KT = weigh_keys(sizeof(T), D), KA = KT / 16;
  __shared__ float part[4 * KT];
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.n_kv;
  const Tiles<KT> tiles(a, tab);
  const int2 at = tiles.find(blockIdx.x / a.n_kv);     // (-1: fewer tiles than there is room for)
  const int s = at.x, k0 = at.y * KT;
  if (s < 0) return;
  const Queries qs = queries_of(a, tab, s);
  const int len = seq_len(a.seqs, s), n = min(len, a.seqs.max_len);
  KeyTile<T, D, KT> keys;
  keys.load(a, s, head, k0, n);
  const bool bad = keys.bad();
  float sum[KA * 4];
#pragma unroll
  for (int x = 0; x < KA * 4; ++x) sum[x] = 0.f;
  const int n_rows = qs.nq * a.group;
  int r0 = wave * 16;
  if (!a.hi) r0 += max(0, k0 - (len - qs.nq)) * a.group / 16 * 16;   // causal: from query k0 on
  for (; r0 < n_rows; r0 += 64) {
    const int r = min(r0 + c16, n_rows - 1), i = r / a.group, gr = r - i * a.group;
    RowInfo row = row_info(a, len, qs, head, i, gr);
    if (r0 + c16 >= n_rows) row.hi = row.lo = 0;
    if (!__any(row.lo < row.hi && row.lo < k0 + KT && row.hi > k0)) continue;
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(qs.tok0 + i) * a.q_token +
                  (int64_t)(head * a.group + gr) * a.q_head;
    frag qf[QF];
#pragma unroll
    for (int kk = 0; kk < QF; ++kk) qf[kk] = load_frag<T, frag>(qp + kk * KSTEP + g * KPL);
    const bool whole = !bad && __all(row.lo <= k0 && row.hi >= k0 + KT);
    add_rows<T, D, KT>(a, a.cap_log2 > 0.f || a.bias, keys, k0, qf, row, whole, sum);
  }
  const float mine = sum_to_lane(sum, c16);
  const int id = c16 % (KA * 4), key = (id >> 2) * 16 + 4 * g + (id & 3);
  if (c16 < KA * 4) part[wave * KT + key] = mine;
  __syncthreads();
  const int j = threadIdx.x;
  if (j < KT && k0 + j < n)
    a.weights.data[(int64_t)s * a.weights.seq + (int64_t)head * a.weights.head + k0 + j] +=
        (part[j] + part[KT + j]) + (part[2 * KT + j] + part[3 * KT + j]);
}

// ---- many rows: queries and what their rows bring go through LDS, for 2 x KT keys of
// a workgroup; two waves hold the same keys and take every other half of a chunk's rows.
// The chunk after the one that is worked on is on its way meanwhile.  8,192 queries over
// 12,288 slots, 32 query and 8 KV heads of 128: 805 us, 683 TFLOP/s (rows from memory,
// without LDS: 1,421 us).  By the counters 7.4 vector instructions go with a matrix
// instruction; the arithmetic of its scores (a fused multiply-add, an exponential, a fused
// multiply-add into the sum) is 3 of them, the others decide who sees what, unpack the
// rows' information and form addresses.  They fill some 45% of the issue, the matrix
// instructions 28%, and waves wait 33% of their time: no limit is reached.  Capped scores
// take 1,716 us, slopes 1,086, documents' intervals 1,066 (165 TFLOP/s of what is seen);
// fp32, 2,048 queries over 4,096 slots of the same heads 735 us, 70 TFLOP/s.
//
// Rows of all sequences, KV head by KV head: info[head][tok0 * group + r].
__global__ __launch_bounds__(256) void weigh_info_kernel(WeighArgs a, WeighTable tab) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.n_tokens * a.group;
  if (idx >= rows * a.n_kv) return;
  const int head = (int)(idx / rows);
  const int at = (int)(idx - head * rows), t = at / a.group;
  int s;
  if (!a.ragged) {
    s = t / a.q_per_seq;
  } else {
    int lo = 0, hi = a.seqs.n_seqs;        // the last sequence that begins at or before t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((a.q_off ? a.q_off[mid] : tab.q[mid]) <= t) lo = mid; else hi = mid;
    }
    s = lo;
  }
  const Queries qs = queries_of(a, tab, s);
  a.info[idx] = row_info(a, seq_len(a.seqs, s), qs, head, t - qs.tok0, at - t * a.group);
}

template <typename T, int D>
struct WideCfg {
  static constexpr int KT = weigh_keys(sizeof(T), D), KEYS = 2 * KT;   // of a wave, of a workgroup
  static constexpr int RB = tile_row_bytes(D * (int)sizeof(T)), CPR = RB / 16, RPW = 1024 / RB;
  static constexpr int ROWS = RB <= 256 ? 64 : 32;                     // of a chunk
  static constexpr int ROUNDS = ROWS * RB / 4096;                      // transfers per wave
  static constexpr int STAGE = ROWS * (RB + (int)sizeof(RowInfo));
  static constexpr int RESIDENT = sizeof(T) == 2 || D <= 96 ? 3 : 2;    // workgroups of a CU
  static_assert(ROUNDS >= 1 && RPW >= 1 && sizeof(RowInfo) == 32, "chunks");
};
// Parts that the rows of every tile are split into, so that few tiles fill the chip.
__device__ __forceinline__ int wide_parts(const WeighArgs& a, long long tiles) {
  return a.slots ? (int)max(1ll, a.slots / (max(tiles, 1ll) * a.n_kv)) : 1;
}

template <typename T, int D, bool GENERAL>
__global__ __launch_bounds__(256, (WideCfg<T, D>::RESIDENT)) void weigh_wide_kernel(WeighArgs a, WeighTable tab) {
  using C = WideCfg<T, D>;
  using MM = Mma16<T>;
  using frag = typename MM::frag;
  constexpr int KPL = MM::KPL, KSTEP = MM::KSTEP, QF = D / KSTEP, KT = C::KT, KA = KT / 16, RB = C::RB;
  __shared__ __align__(1024) char lds[2 * C::STAGE];
  __shared__ float part[2 * C::KEYS];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave & 1, rg = wave >> 1;
  for (long long u = blockIdx.x;; u += gridDim.x) {
    const Tiles<C::KEYS> tiles(a, tab);           // (not kept in registers through the rows)
    const int parts = wide_parts(a, tiles.total);
    if (u >= tiles.total * a.n_kv * parts) return;
    const int head = (int)(u % a.n_kv);
    const long long tp = u / a.n_kv;
    const int p = (int)(tp / tiles.total);
    const int2 at = tiles.find(tp - p * tiles.total);
    const int s = at.x;
    if (s < 0) return;
    const Queries qs = queries_of(a, tab, s);
    const int len = seq_len(a.seqs, s), n = min(len, a.seqs.max_len);
    const int kw = at.y * C::KEYS, k0 = kw + kg * KT;     // the workgroup's, the wave's first key
    KeyTile<T, D, KT> keys;
    keys.load(a, s, head, min(k0, n - 1), n);
    const bool bad = keys.bad();
    float sum[KA * 4];
#pragma unroll
    for (int x = 0; x < KA * 4; ++x) sum[x] = 0.f;
    // ---- this part's chunks of rows
    const int n_rows = qs.nq * a.group;
    int r0 = 0;
    if (!a.hi) r0 = max(0, kw - (len - qs.nq)) * a.group / C::ROWS * C::ROWS;   // causal
    const int chunks = (n_rows - r0 + C::ROWS - 1) / C::ROWS, per = (chunks + parts - 1) / parts;
    const int c0 = min(p * per, chunks), c1 = min(c0 + per, chunks);
    r0 += c0 * C::ROWS;
    const char* qbase = static_cast<const char*>(a.q) +
                        ((int64_t)qs.tok0 * a.q_token + (int64_t)head * a.group * a.q_head) * (int)sizeof(T);
    const RowInfo* info = a.info + ((int64_t)head * a.n_tokens + qs.tok0) * a.group;
    // Where a round's rows are whole queries, a lane's query and head of the group are the
    // same in every round, and the rest of its address is the same for all lanes.
    constexpr int STEP = 4 * C::RPW;                      // rows of a round
    const uint32_t qt = (uint32_t)(a.q_token * (int64_t)sizeof(T)), qh = (uint32_t)(a.q_head * (int64_t)sizeof(T));
    const bool steps = RB <= 256 && STEP % a.group == 0 && a.near;
    uint32_t lane_at;
    {
      const int row = wave * C::RPW + lane_again() / C::CPR, i = row / a.group;
      int ch = (lane_again() % C::CPR) ^ row_swizzle<RB>(row);
      if (D * (int)sizeof(T) < RB && ch * 16 >= D * (int)sizeof(T)) ch = 0;   // (never read)
      lane_at = (uint32_t)i * qt + (uint32_t)(row - i * a.group) * qh + ch * 16;   // (used where `near`)
    }
    auto issue = [&](int first, int st) {                 // rows from `first` on into stage st
      char* base = lds + st * C::STAGE;
      if (steps && first + C::ROWS <= n_rows) {
        const char* from = qbase + (int64_t)(first / a.group) * a.q_token * (int)sizeof(T);
#pragma unroll
        for (int r = 0; r < C::ROUNDS; ++r) {
          dma16(from + lane_at, base + (r * 4 + wave) * 1024);
          from += (int64_t)(STEP / a.group) * a.q_token * (int)sizeof(T);
        }
      } else {
        const int lane = lane_again();
#pragma unroll 1
        for (int r = 0; r < C::ROUNDS; ++r) {
          const int row = (r * 4 + wave) * C::RPW + lane / C::CPR;
          int ch = (lane % C::CPR) ^ row_swizzle<RB>(row);
          if (D * (int)sizeof(T) < RB && ch * 16 >= D * (int)sizeof(T)) ch = 0;
          const int x = min(first + row, n_rows - 1), i = x / a.group;
          dma16(qbase + ((int64_t)i * a.q_token + (int64_t)(x - i * a.group) * a.q_head) * (int)sizeof(T) + ch * 16,
                base + (r * 4 + wave) * 1024);
        }
      }
      if (wave < C::ROWS / 32) {
        const int lane = lane_again();                    // (a row past the last one is not looked at)
        dma16(reinterpret_cast<const char*>(info + min(first + wave * 32 + lane / 2, n_rows - 1)) + lane % 2 * 16,
              base + C::ROWS * RB + wave * 1024);
      }
    };
    if (c0 < c1) issue(r0, 0);
    for (int c = c0; c < c1; ++c, r0 += C::ROWS) {
      const int st = (c - c0) & 1;
      wait_vmcnt<0>();
      __syncthreads();                                    // this chunk is there, the other stage idle
      if (c + 1 < c1) issue(r0 + C::ROWS, st ^ 1);
      const char* base = lds + st * C::STAGE;
      const RowInfo* ri = reinterpret_cast<const RowInfo*>(base + C::ROWS * RB);
#pragma unroll 1
      for (int h = 0; h < C::ROWS / 32; ++h) {
        const int lane = lane_again(), rr = (h * 2 + rg) * 16 + (lane & 15);
        RowInfo row;
        const int4 w = *reinterpret_cast<const int4*>(ri + rr);
        row.lo = w.x;
        row.hi = r0 + rr < n_rows ? w.y : 0;
        row.ref = __int_as_float(w.z);
        row.factor = __int_as_float(w.w);
        if (!__any(row.lo < row.hi && row.lo < k0 + KT && row.hi > k0)) continue;
        if (GENERAL) {
          row.p = ri[rr].p;
          row.slope = ri[rr].slope;
        }
        frag qf[QF];
#pragma unroll
        for (int kk = 0; kk < QF; ++kk) {
          const int byte = (kk * KSTEP + (lane >> 4) * KPL) * (int)sizeof(T);
          qf[kk] = *reinterpret_cast<const frag*>(base + row_offset<RB>(rr, byte >> 4));
        }
        const bool whole = !bad && __all(row.lo <= k0 && row.hi >= k0 + KT);
        add_rows<T, D, KT>(a, GENERAL, keys, k0, qf, row, whole, sum);
      }
    }
    const int c16 = lane_again() & 15, g = lane_again() >> 4;
    const float mine = sum_to_lane(sum, c16);
    const int id = c16 % (KA * 4), key = kg * KT + (id >> 2) * 16 + 4 * g + (id & 3);
    __syncthreads();
    if (c16 < KA * 4) part[rg * C::KEYS + key] = mine;
    __syncthreads();
    if (tid < C::KEYS && kw + tid < n) {
      const float v = part[tid] + part[C::KEYS + tid];
      if (parts == 1)
        a.weights.data[(int64_t)s * a.weights.seq + (int64_t)head * a.weights.head + kw + tid] += v;
      else
        a.partial[u * C::KEYS + tid] = v;
    }
    __syncthreads();
  }
}

// Adds the parts of every tile to the weights, in order.
template <int KEYS>
__global__ __launch_bounds__(KEYS < 64 ? 64 : KEYS) void weigh_merge_kernel(WeighArgs a, WeighTable tab) {
  const Tiles<KEYS> tiles(a, tab);
  const int parts = wide_parts(a, tiles.total);
  if (parts == 1) return;
  const int head = blockIdx.x % a.n_kv, t = blockIdx.x / a.n_kv, j = threadIdx.x;
  if (t >= tiles.total) return;
  const int2 at = tiles.find(t);
  if (at.x < 0 || j >= KEYS) return;
  const int key = at.y * KEYS + j;
  if (key >= min(seq_len(a.seqs, at.x), a.seqs.max_len)) return;
  float v = 0.f;
  for (int p = 0; p < parts; ++p) v += a.partial[((p * tiles.total + t) * a.n_kv + head) * KEYS + j];
  a.weights.data[(int64_t)at.x * a.weights.seq + (int64_t)head * a.weights.head + key] += v;
}

template <typename T, int D>
hipError_t weigh_as(const WeighArgs& a, const WeighTable& tab, hipStream_t s) {
  if (a.kind == kWeighToken) {
    // as many waves as there can be tiles, about sixteen to a CU
    const int64_t groups = (weigh_tiles(a, weigh_token_keys(sizeof(T), D)) + 3) / 4;
    const int64_t most = (1024 + a.n_kv - 1) / a.n_kv;
    const dim3 grid((unsigned)(a.n_kv * (groups < most ? groups : most)));
    CR_LAUNCH((weigh_token_kernel<T, D>), grid, dim3(256), 0, s, a, tab);
  } else if (a.kind == kWeighRows) {
    const dim3 grid((unsigned)(weigh_tiles(a, weigh_keys(sizeof(T), D)) * a.n_kv));   // (at most kWeighSlots)
    CR_LAUNCH((weigh_rows_kernel<T, D>), grid, dim3(256), 0, s, a, tab);
  } else {
    constexpr int KEYS = WideCfg<T, D>::KEYS;
    const int64_t rows = (int64_t)a.n_tokens * a.group * a.n_kv;
    CR_LAUNCH(weigh_info_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, s, a, tab);
    const int64_t groups = a.slots ? a.slots : weigh_tiles(a, KEYS) * a.n_kv;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192));
    if (a.cap_log2 > 0.f || a.bias) {
      CR_LAUNCH((weigh_wide_kernel<T, D, true>), grid, dim3(256), 0, s, a, tab);
    } else {
      CR_LAUNCH((weigh_wide_kernel<T, D, false>), grid, dim3(256), 0, s, a, tab);
    }
    if (a.slots) {
      const dim3 tiles((unsigned)(weigh_tiles(a, KEYS) * a.n_kv));
      CR_LAUNCH((weigh_merge_kernel<KEYS>), tiles, dim3(KEYS < 64 ? 64 : KEYS), 0, s, a, tab);
    }
  }
  return hipGetLastError();
}

template <typename T>
hipError_t weigh(const WeighArgs& a, const WeighTable& tab, hipStream_t s) {
  switch (a.head_dim) {
    case 32: return weigh_as<T, 32>(a, tab, s);
    case 64: return weigh_as<T, 64>(a, tab, s);
    case 96: return weigh_as<T, 96>(a, tab, s);
    case 128: return weigh_as<T, 128>(a, tab, s);
    case 160: return weigh_as<T, 160>(a, tab, s);
    case 192: return weigh_as<T, 192>(a, tab, s);
    case 224: return weigh_as<T, 224>(a, tab, s);
    case 256: return weigh_as<T, 256>(a, tab, s);
    default: return hipErrorInvalidValue;
  }
}
template hipError_t weigh<bf16>(const WeighArgs&, const WeighTable&, hipStream_t);
template hipError_t weigh<float>(const WeighArgs&, const WeighTable&, hipStream_t);

}  // namespace cr
