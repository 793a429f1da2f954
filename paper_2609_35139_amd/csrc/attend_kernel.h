// Attention from new queries to a paged cache (gfx950 MFMA).
//
// Row (t, h) of query t and head h sees the positions j of its sequence with
// lo(t) <= j < hi(t); hi is t's own position + 1 unless the caller gives it:
//   x_j = scale * q.k_j;  x_j = cap * tanh(x_j / cap);  x_j -= slope_h |p_t - j|
//   o = sum_j exp(x_j - m) v_j / l,  l = sum_j exp(x_j - m),  lse = m + log l.
// A row that sees nothing has o = 0 and lse = -inf.
//
// The heads of a group share their keys, so a workgroup's tile packs rows
// (query, head of the group) of one sequence and one KV head: row r is query
// r / group.  A tile walks its keys once with a running maximum and sum; where
// there are few tiles the keys are split among several workgroups, whose
// (max, sum, unnormalised o) a second kernel joins.  The lengths are known on
// the device alone (a captured launch is replayed as they grow), so every
// workgroup derives the split from them, see plan_item.
//
// Keys and values are staged in LDS as they lie in the pages (16-byte
// global->LDS transfers whose addresses come from the block list of the
// segment, itself in LDS).  Scores are formed transposed, S^T = K Q^T, in
// 16x16 atoms: a lane holds four consecutive keys of one row, so maximum and
// sum are register work plus two exchanges, and the probabilities are already
// the B operand of O^T = V^T P^T.  Its A operand needs four consecutive keys
// of one dim per lane: for bf16 the LDS reads that transpose 16-bit elements
// deliver that from the row-major tile.
//
// What it reaches (a large copy runs at 5.1 TB/s, a large product at 1,250
// TFLOP/s in bf16 and 144 in fp32):
//  - one token per sequence, rows of 16: bound by reading keys and values, 64
//    sequences of 64 to 16,000 keys (716 MB) in 148 us, 4.8 TB/s; 4 of 131,072
//    (513 MB) in 98 us, 5.2 TB/s.  Of a single one of 4,096 keys (14 us with the
//    merge) most is the chain of dependent reads and the second launch.
//  - long prompts, wide units: bound by the waves' own instructions, the matrix
//    pipes work 43% of the time; 8,192 queries over 12,288 keys, 32 heads of 128
//    in 1,100 us, 1,000 TFLOP/s.
//  - in between (8 to 300 queries a sequence), the parts' partial results and
//    uneven rounds cost as much as the products; see attend_plan.
#pragma once
#include <climits>
#include <type_traits>

#include "serve.h"

namespace cr {

constexpr int kPlanTile = 64;     // keys per tile of the split's arithmetic
constexpr int kListPages = 512;   // pages of a segment's block list
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kMostSum = 16777216.f;   // 2^24: a lane's share of a tile's probabilities

// ------------------------------------------------------------ units and rows
// A sequence's length: its queries' slots count from it, but keys lie only in
// slots below max_len.
__device__ __forceinline__ int seq_len(const PagedSeqs& p, int s) { return max(p.lens[s], 0); }
// The offsets of a ragged batch.
struct Offsets {
  const AttendArgs& a;
  const SeqTable& t;
  __device__ __forceinline__ int q(int i) const { return a.q_off ? a.q_off[i] : t.q[i]; }
  __device__ __forceinline__ int unit(int i) const { return a.unit_off ? a.unit_off[i] : t.unit[i]; }
  // the sequence (the last one that begins at or before it) of a query or unit
  template <typename F>
  __device__ __forceinline__ int find(F&& off, int x) const {
    int lo = 0, hi = a.seqs.n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (off(mid) <= x) lo = mid; else hi = mid;
    }
    return lo;
  }
  __device__ __forceinline__ int of_query(int t) const {
    return find([&](int i) { return q(i); }, t);
  }
  __device__ __forceinline__ int of_unit(int u) const {
    return find([&](int i) { return unit(i); }, u);
  }
};
struct Unit {
  int s, tile;       // sequence and its row tile
  int tok0, nq;      // the sequence's first query and number of queries
};
__device__ __forceinline__ Unit unit_of(const AttendArgs& a, const SeqTable& tab, int u) {
  Unit x;
  if (a.ragged) {
    const Offsets off{a, tab};
    x.s = off.of_unit(u);
    x.tile = u - off.unit(x.s);
    x.tok0 = off.q(x.s);
    x.nq = off.q(x.s + 1) - x.tok0;
  } else {
    x.s = u / a.units_per_seq;
    x.tile = u - x.s * a.units_per_seq;
    x.tok0 = x.s * a.q_per_seq;
    x.nq = a.q_per_seq;
  }
  return x;
}
// One past the last position that a unit's queries may see.
__device__ __forceinline__ int unit_end(const AttendArgs& a, const Unit& x) {
  const int n = seq_len(a.seqs, x.s);
  if (a.hi) return min(n, a.seqs.max_len);
  const int last = min(((x.tile + 1) * a.rows - 1) / a.group, x.nq - 1);
  return min(n - (x.nq - 1 - last), a.seqs.max_len);
}
__device__ __forceinline__ int unit_tiles(const AttendArgs& a, const SeqTable& tab, int u) {
  return (max(unit_end(a, unit_of(a, tab, u)) - a.key_begin, 0) + kPlanTile - 1) / kPlanTile;
}
// Positions [lo, hi) that query i of a sequence (token t) sees in this pass.
__device__ __forceinline__ int2 interval_of(const AttendArgs& a, int n, int nq, int i, int t) {
  const int most = min(n, a.seqs.max_len);
  int hi = max(min(a.hi ? a.hi[t] : n - nq + i + 1, most), 0);   // (differences stay in 32 bits)
  int lo = a.lo ? max(a.lo[t], 0) : 0;
  if (a.shared) hi = min(hi, a.shared);
  else lo = max(lo, a.key_begin);
  return make_int2(lo, hi);
}

// ------------------------------------------------------------------- split
// Item `it` of the split: unit, part, number of the unit's parts, tiles per
// part, and the unit's first item (all uniform).  Every unit has at least one
// part; a part is `chunk` tiles, the mean load of a.slots workgroups, so there
// are at most a.slots + n_units items.  The same in every wave of every
// workgroup.
struct Item { int unit, part, parts, chunk, first; };
__device__ __forceinline__ int div_up(int t, int chunk) {
  return (int)(((unsigned)t + (unsigned)chunk - 1u) / (unsigned)chunk);
}
__device__ __forceinline__ Item plan_item(const AttendArgs& a, const SeqTable& tab, int it) {
  const int lane = threadIdx.x & 63;
  const int U = a.n_units;
  const int t0 = lane < U ? unit_tiles(a, tab, lane) : 0;   // the first 64 units stay in registers
  auto tiles = [&](int u0) {
    return u0 == 0 ? t0 : (u0 + lane < U ? unit_tiles(a, tab, u0 + lane) : 0);
  };
  // (sums in fp32: a chunk need not be exact, only the same everywhere)
  float total = 0.f;
  for (int u0 = 0; u0 < U; u0 += 64) total += wave_sum((float)tiles(u0));
  int chunk = max(a.min_tiles, (int)fminf(total / (float)a.slots + 1.f, 1e9f));
  // a few units: longer parts, until they are at most a.slots
  for (int k = 0; k < 8 && U > 1 && U <= a.one_round; ++k) {
    float cnt = 0.f;
    for (int u0 = 0; u0 < U; u0 += 64)
      cnt += wave_sum(u0 + lane < U ? (float)max(1, div_up(tiles(u0), chunk)) : 0.f);
    if (cnt <= (float)a.slots) break;
    chunk += max(1, (int)((float)chunk * (cnt / (float)a.slots - 1.f) * 0.7f));
  }
  if (a.split_cost > 0.f) {
    const int limit = (int)fminf((float)chunk * a.split_cost + a.join_cost, 1e9f);
    bool longer = false;
    for (int u0 = 0; u0 < U; u0 += 64) longer |= __any(tiles(u0) > limit);
    if (!longer) chunk = limit;
  }
  chunk = __builtin_amdgcn_readfirstlane(chunk);
  Item r{-1, 0, 1, chunk, 0};
  int base = 0;
  for (int u0 = 0; u0 < U; u0 += 64) {
    const int n = u0 + lane < U ? max(1, div_up(tiles(u0), chunk)) : 0;
    int incl = n;
    if (U > 1) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(incl, o);
        if (lane >= o) incl += x;
      }
    }
    const unsigned long long hit = __ballot(n > 0 && base + incl > it);
    if (hit) {
      const int l = __ffsll(hit) - 1;
      r.unit = u0 + l;
      r.parts = __builtin_amdgcn_readlane(n, l);
      r.first = base + __builtin_amdgcn_readlane(incl, l) - r.parts;
      r.part = it - r.first;
      break;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return r;
}

// ------------------------------------------------------------- type specifics
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Rows of RB bytes in 16-byte chunks; chunk c of row r lies in slot
// c ^ f(r), f periodic in 16 rows, so that the 16 rows of a fragment read and
// the four rows of a transposing read start in distinct banks.
constexpr int tile_row_bytes(int bytes) {
  int r = 64;
  while (r < bytes) r *= 2;
  return r;
}
template <int RB>
__device__ __forceinline__ int row_swizzle(int row) {
  constexpr int CPR = RB / 16;
  if constexpr (RB >= 256) return row & 15;
  else return (row / (256 / RB)) & (CPR - 1);
}
template <int RB>
__device__ __forceinline__ int row_offset(int row, int chunk) {
  return row * RB + ((chunk ^ row_swizzle<RB>(row)) << 4);
}

// A capped score is cap * tanh(u), u = score / cap.  For |u| <= 1/2 that is
// score * tanh(u) / u, the quotient a polynomial in u^2: the error is relative to
// the score however large the cap (2^-23; a cap times a tanh that is off by 2^-23
// would be off by 0.1 for a cap of a million).  tanh(u) / u - 1 = u^2 (c_0 + c_1
// u^2 + ...), a least-squares fit reweighted towards the largest errors until
// they level out (Lawson's iteration), relative error 2^-26.
constexpr float kCapSmall = 0.5f;
constexpr float kCapPoly[4] = {-0.333331435918808f, 0.13325878977775574f, -0.05304549261927605f,
                               0.01724149100482464f};
__device__ __forceinline__ float tanh_over(float u) {
  const float w = u * u;
  float p = kCapPoly[3];
#pragma unroll
  for (int k = 2; k >= 0; --k) p = __builtin_fmaf(p, w, kCapPoly[k]);
  return __builtin_fmaf(p, w, 1.f);
}
// tanh(x) for |x| > 1/2: for bf16 through one exponential and a reciprocal
// (relative error up to 2^-20, as large as that of a score's fp32 sum over 16
// dims), for fp32 the library's.
template <typename T> __device__ __forceinline__ float tanh_of(float x);
template <> __device__ __forceinline__ float tanh_of<float>(float x) { return tanhf(x); }
template <> __device__ __forceinline__ float tanh_of<bf16>(float x) {
  const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2e));   // inf for large x: 1 - 0
  return 1.f - 2.f * __builtin_amdgcn_rcpf(e + 1.f);
}

// Keys of a PV atom, its V fragment from the row-major tile, and a fragment's
// finite values and indicators of the others.
template <typename T> struct ValueOps;
template <> struct ValueOps<bf16> {
  typedef bf16x8 frag;
  static constexpr int KEYS = 32;       // keys contracted by one atom: two 16-key sub-tiles
  // lane (g, i): dims d0 + i, keys key0 + 4 g + [0, 4) and key0 + 16 + 4 g + [0, 4).
  // A transposing read takes 8 bytes per lane: of 16 lanes, lanes 4 r .. 4 r + 3
  // hold row r's 16 elements and lane i receives element i of the four rows.
  template <int RB>
  __device__ __forceinline__ static frag load(const char* tile, int key0, int d0, int lane) {
    const int i = lane & 15, g = lane >> 4;
    const int row = key0 + 4 * g + (i >> 2);
    const int byte = (d0 + (i & 3) * 4) * 2;
    const char* p = tile + row_offset<RB>(row, byte >> 4) + (byte & 15);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * RB));
    frag r;
    *reinterpret_cast<s16x4*>(&r) = lo;
    *(reinterpret_cast<s16x4*>(&r) + 1) = hi;
    return r;
  }
  // (two elements to a word; without compares, whose masks would fill the
  // scalar registers)
  // 1 in each half that is infinite or NaN
  __device__ __forceinline__ static uint32_t not_finite(uint32_t w) {
    return (((w & 0x7fff7fffu) + 0x00800080u) >> 15) & 0x00010001u;
  }
  __device__ __forceinline__ static uint32_t odd_bits(const frag& v) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    return (not_finite(w[0]) | not_finite(w[1])) | (not_finite(w[2]) | not_finite(w[3]));
  }
  __device__ __forceinline__ static frag finite_part(const frag& v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t m = not_finite(w[i]);
      w[i] &= ~((m << 16) - m);       // 0xffff in each such half
    }
    return __builtin_bit_cast(frag, w);
  }
  // 1.0 where the value is infinite with this sign (0 +, 1 -) or NaN
  __device__ __forceinline__ static frag odd_part(const frag& v, int sign) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t nan = (((w[i] & 0x7fff7fffu) + 0x007f007fu) >> 15) & 0x00010001u;
      const uint32_t neg = (w[i] >> 15) & 0x00010001u;
      const uint32_t m = nan | (not_finite(w[i]) & (sign ? neg : ~neg));
      w[i] = (m << 14) - (m << 7);    // 0x3f80 in each such half
    }
    return __builtin_bit_cast(frag, w);
  }
};
template <> struct ValueOps<float> {
  typedef f32x4 frag;
  static constexpr int KEYS = 16;
  template <int RB>
  __device__ __forceinline__ static frag load(const char* tile, int key0, int d0, int lane) {
    const int d = d0 + (lane & 15), g = lane >> 4;
    frag r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = key0 + 4 * g + e;
      r[e] = *reinterpret_cast<const float*>(tile + row_offset<RB>(row, d >> 2) + (d & 3) * 4);
    }
    return r;
  }
  __device__ __forceinline__ static uint32_t not_finite(uint32_t w) {
    return ((w & 0x7fffffffu) + 0x00800000u) >> 31;
  }
  __device__ __forceinline__ static uint32_t odd_bits(const frag& v) {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    return (not_finite(w[0]) | not_finite(w[1])) | (not_finite(w[2]) | not_finite(w[3]));
  }
  __device__ __forceinline__ static frag finite_part(const frag& v) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= not_finite(w[i]) - 1u;
    return __builtin_bit_cast(frag, w);
  }
  __device__ __forceinline__ static frag odd_part(const frag& v, int sign) {
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t nan = ((w[i] & 0x7fffffffu) + 0x007fffffu) >> 31, neg = w[i] >> 31;
      w[i] = (nan | (not_finite(w[i]) & (sign ? neg : neg ^ 1u))) * 0x3f800000u;
    }
    return __builtin_bit_cast(frag, w);
  }
};

// maximum and sum over the four lanes that hold one row (l, l^16, l^32, l^48)
__device__ __forceinline__ float row_max(float x) {
  const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_max(fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1])));
}
__device__ __forceinline__ float row_sum(float x) {
  const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return halves_sum(__uint_as_float(v[0]) + __uint_as_float(v[1]));
}

// This lane's number, from no register that has to live.  (opaque: not merged
// with an earlier one)
__device__ __forceinline__ int lane_again() {
  int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(l));
  return l;
}

// ------------------------------------------------------------------ kernel
// RG * KG waves: KG groups of RG waves walk alternate tiles of KT keys, each
// with its own ring of STAGES tiles; the RG waves of a group own 16 * NQ rows
// each.
template <typename T, int D, int NQ, int RG, int KG, int KT, int STAGES>
struct AttendCfg {
  static constexpr int WAVES = RG * KG, NT = 64 * WAVES, ROWS = 16 * NQ * RG;
  static constexpr int RB = tile_row_bytes(D * (int)sizeof(T)), CPR = RB / 16, RPW = 1024 / RB;
  static constexpr int TILE = KT * RB;                    // bytes of a K or V tile
  static constexpr int ROUNDS = TILE / (RG * 1024);       // transfers per wave and tile
  static constexpr int RING = STAGES * 2 * TILE;
  static constexpr int MLD = D + 4;                      // merge rows, in floats
  static constexpr int MERGE = KG > 1 ? KG * ROWS * (MLD + 2) * 4 : 0;
  static constexpr int LDS = KG * RING > MERGE ? KG * RING : MERGE;
  static_assert(ROUNDS * RG * 1024 == TILE && RPW >= 1 && KT % ValueOps<T>::KEYS == 0, "tile");
  static constexpr int BYTES = LDS + kListPages * 8 + kListPages / 8 + 16 + ROWS * 16;
  static_assert(BYTES <= 160 * 1024 && ROWS <= NT, "LDS");
  static_assert(2 * ROUNDS * (STAGES - 1) < 64, "transfers in flight");
  static_assert(KT <= 128 && KT * KG < kListPages, "bits of a lane's scores, keys of a list");
};

template <typename T, int D, int NQ, int RG, int KG, int KT, int STAGES, int OCC = 1>
__global__ __launch_bounds__(64 * RG * KG, OCC) void attend_kernel(AttendArgs a, SeqTable tab) {
  using C = AttendCfg<T, D, NQ, RG, KG, KT, STAGES>;
  using MM = Mma16<T>;
  using VO = ValueOps<T>;
  using frag = typename MM::frag;
  constexpr int KPL = MM::KPL, KSTEP = MM::KSTEP;
  // a wave works on KS keys of a tile at a time
  constexpr int KS = VO::KEYS;
  constexpr int QF = D / KSTEP, DT = D / 16, ST = KS / 16, PF = KS / VO::KEYS;
  constexpr int RB = C::RB;
  // The matrix instructions take bf16 probabilities.  Units of 16 rows, bound by
  // reading the keys, multiply V by what that leaves over too (16 bits in all, an
  // error of 0.0017 instead of 0.0020 of the output, bf16's own rounding 0.0017;
  // 148 us with and without for 64 sequences of 64 to 16,000 keys of 128 dims, 242
  // and 235 for 32 of 2,000 to 8,000 of 256).  Wide units round to bf16 (8,192
  // queries over 12,288 keys would take 1,619 instead of 1,137 us, 590 tokens of
  // questions 93 instead of 65); their sum is then of the rounded ones, so that the
  // weights still add up to one.
  constexpr bool FINE = sizeof(T) == 2 && RG == 1;
  constexpr int PL = FINE ? PF : 1;
  constexpr int VE = NQ > 1 && sizeof(T) == 2 && D >= 64 && D <= 128 ? 3 : 0;
  // rings (later the merge area), the segment's block list (addresses of the
  // blocks' keys), the bits of those that are no block, and of every row (lo,
  // hi, p, slope): one array, since the compiler waits for every transfer in
  // flight before it reads LDS where it tells several apart
  __shared__ __align__(1024) char lds[C::BYTES];
  uint64_t* const list = reinterpret_cast<uint64_t*>(lds + C::LDS);
  uint32_t* const none = reinterpret_cast<uint32_t*>(list + kListPages);
  int4* const info = reinterpret_cast<int4*>(none + kListPages / 32 + 4);

  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / RG, rg = wave % RG;
  const int head = blockIdx.x % a.n_kv;                    // KV head
  const int item = blockIdx.x / a.n_kv;

  // ---- the item's unit, rows and keys
  int unit = item, part = 0, parts = 1, chunk = 0, slot = item;
  if (a.shared) {
    unit = item / a.splits;
    part = item - unit * a.splits;
    chunk = a.split_tiles;
  } else if (a.slots) {
    const Item p = plan_item(a, tab, item);
    if (p.unit < 0) return;
    unit = p.unit; part = p.part; parts = p.parts; chunk = p.chunk;
    if (part == 0 && head == 0 && tid == 0) a.unit_items[unit] = make_int2(p.first, p.parts);
  } else if (a.always_partial && head == 0 && tid == 0) {
    a.unit_items[unit] = make_int2(unit, 1);
  }
  Unit x{0, unit, 0, a.n_tokens};
  if (!a.shared) x = unit_of(a, tab, unit);
  x.s = __builtin_amdgcn_readfirstlane(x.s);
  x.tile = __builtin_amdgcn_readfirstlane(x.tile);
  x.tok0 = __builtin_amdgcn_readfirstlane(x.tok0);
  x.nq = __builtin_amdgcn_readfirstlane(x.nq);
  const int row0 = x.tile * C::ROWS, n_rows = min(C::ROWS, x.nq * a.group - row0);
  const int seq_n = a.shared ? 0 : seq_len(a.seqs, x.s);
  // this lane's rows, on their way from here
  frag qf[NQ][QF];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = (rg * NQ + n) * 16 + c16;
    const int i = (row0 + min(r, n_rows - 1)) / a.group;
    const T* qp = static_cast<const T*>(a.q) + (int64_t)(x.tok0 + i) * a.q_token +
                  (int64_t)(head * a.group + row0 + min(r, n_rows - 1) - i * a.group) * a.q_head;
#pragma unroll
    for (int kk = 0; kk < QF; ++kk)
      qf[n][kk] = r < n_rows ? load_frag<T, frag>(qp + kk * KSTEP + g * KPL) : frag{};
  }
  // position and interval of every row of the unit, and the keys that any row
  // sees (a row past the last one sees everything: it masks nothing)
  if (tid < C::ROWS) {
    int4 w{0, INT_MAX, 0, 0};
    if (tid < n_rows) {
      const int i = (row0 + tid) / a.group;
      int n = seq_n, nq = x.nq, qi = i;
      if (a.shared) {
        const Offsets off{a, tab};
        const int s = a.ragged ? off.of_query(i) : i / a.q_per_seq;
        const int o = a.ragged ? off.q(s) : s * a.q_per_seq;
        nq = a.ragged ? off.q(s + 1) - o : a.q_per_seq;
        n = seq_len(a.seqs, s);
        qi = i - o;
      }
      const int2 iv = interval_of(a, n, nq, qi, x.tok0 + i);
      const float slope = a.bias ? a.slopes_log2[head * a.group + row0 + tid - i * a.group] : 0.f;
      w = int4{iv.x, iv.y, n - nq + qi, __float_as_int(slope)};
    }
    info[tid] = w;
  }
  __syncthreads();
  int kb = INT_MAX, ke = INT_MIN;
  for (int r = lane; r < n_rows; r += 64) {
    const int lo = info[r].x, hi = info[r].y;
    if (lo < hi) { kb = min(kb, lo); ke = max(ke, hi); }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    kb = min(kb, __shfl_xor(kb, o));
    ke = max(ke, __shfl_xor(ke, o));
  }
  if (chunk) {
    const int64_t b = (int64_t)a.key_begin + (int64_t)part * chunk * kPlanTile;
    kb = (int)max((int64_t)kb, b);
    // (the last part of a planned unit takes whatever is left)
    if (a.shared || part + 1 < parts) ke = (int)min((int64_t)ke, b + (int64_t)chunk * kPlanTile);
  }
  kb = __builtin_amdgcn_readfirstlane(kb);
  ke = __builtin_amdgcn_readfirstlane(ke);

  // ---- the window that every row of the wave sees
  int wlo = INT_MIN, whi = INT_MAX;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = (rg * NQ + n) * 16 + c16;
    wlo = max(wlo, info[r].x);
    whi = min(whi, info[r].y);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    wlo = max(wlo, __shfl_xor(wlo, o));
    whi = min(whi, __shfl_xor(whi, o));
  }
  wlo = __builtin_amdgcn_readfirstlane(wlo);
  whi = __builtin_amdgcn_readfirstlane(whi);
  const bool idle = rg * NQ * 16 >= n_rows;     // no row: the wave only stages

  f32x4 oacc[NQ][DT];
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    m[n] = -INFINITY;
    l[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) oacc[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool general = a.cap_log2 > 0.f || a.bias;
  const float cc = general ? 1.f : a.scale_log2;

  const char* kbase = static_cast<const char*>(a.k) + (int64_t)head * a.seqs.head * sizeof(T);
  const uint64_t to_values = (uint64_t)a.v - (uint64_t)a.k;
  const uint32_t token_bytes = (uint32_t)(a.seqs.token * (int64_t)sizeof(T));   // (32 bits: checked on the host)
  char* ring = lds + kg * C::RING;
  const int shift = a.seqs.shift, page_mask = (1 << shift) - 1;
  const int* table = a.seqs.table + (int64_t)x.s * a.seqs.max_blocks;
  constexpr int STEP = KT * KG;
  const int pages = kListPages - 1;       // (a segment may begin inside a page)
  const int seg_most = (pages << shift) / STEP * STEP;

  for (int seg = kb, seg_end; seg < ke; seg = seg_end) {
    // ---- a segment: its block list, then its tiles through the ring
    seg_end = ke - seg <= seg_most ? ke : seg + seg_most;
    const int p0 = seg >> shift, np = ((seg_end - 1) >> shift) - p0 + 1;
    const int tid = wave * 64 + lane_again();   // (not kept in a register through the loops)
    __syncthreads();                       // the last segment's list and ring are idle
    if (tid <= kListPages / 32) none[tid] = 0;    // (the last word: any)
    __syncthreads();
    uint64_t k0 = (uint64_t)kbase;
    asm volatile("" : "+s"(k0));
    for (int i = tid; i < np; i += C::NT) {
      const int id = table[p0 + i];
      const bool ok = id >= 0 && id < a.seqs.n_blocks;
      list[i] = k0 + (ok ? (int64_t)id * a.seqs.block * (int64_t)sizeof(T) : 0);
      if (!ok) {
        atomicOr(none + i / 32, 1u << (i % 32));
        none[kListPages / 32] = 1;
      }
    }
    // (the rows are waited for here: a load still pending at the loops' entry would
    // have every turn of them wait for all transfers in flight)
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int kk = 0; kk < QF; ++kk) asm volatile("" : "+v"(qf[n][kk]));
    __syncthreads();
    const bool seg_bad = __builtin_amdgcn_readfirstlane(none[kListPages / 32]) != 0;
    const int tiles = (seg_end - seg + KT - 1) / KT;
    const int iters = (tiles + KG - 1) / KG, mine = (tiles - kg + KG - 1) / KG;

    auto issue = [&](int i, int st, int lane) {   // tile i of this group into ring slot st
      const int k0 = seg + (i * KG + kg) * KT;
      uint64_t src[C::ROUNDS];
#pragma unroll
      for (int r = 0; r < C::ROUNDS; ++r) {
        const int row = (r * RG + rg) * C::RPW + lane / C::CPR;
        int ch = (lane % C::CPR) ^ row_swizzle<RB>(row);
        if (D * (int)sizeof(T) < RB && ch * 16 >= D * (int)sizeof(T)) ch = 0;   // (never read)
        const int key = min(k0 + row, seg_end - 1);      // never past the last key seen
        src[r] = list[(key >> shift) - p0] + (uint64_t)(uint32_t)(key & page_mask) * token_bytes + ch * 16;
      }
      char* base = ring + st * 2 * C::TILE;
#pragma unroll
      for (int r = 0; r < C::ROUNDS; ++r)
        dma16(reinterpret_cast<const char*>(src[r]), base + (r * RG + rg) * 1024);
#pragma unroll
      for (int r = 0; r < C::ROUNDS; ++r)
        dma16(reinterpret_cast<const char*>(src[r] + to_values), base + C::TILE + (r * RG + rg) * 1024);
    };

    // K fragment (sub-tile t, step kk) of a tile
    auto key_frag = [&](const char* kt, int t, int kk, int lane) {
      const int byte = (kk * KSTEP + (lane >> 4) * KPL) * (int)sizeof(T);
      return *reinterpret_cast<const frag*>(kt + row_offset<RB>(t * 16 + (lane & 15), byte >> 4));
    };
    // scores of row block n in exp2 units, before the mask, where they are not
    // just scaled
    auto transform = [&](f32x4 (&s)[ST], int n, int k0, int lane) {
      if (a.cap_log2 > 0.f) {
        // few scores are past half the cap in earnest: the second form is formed
        // only where a wave has one (the second for every score / as here: 4,096
        // queries over 8,192 keys, cap 30, 700 / 689 us; cap 2, most scores past
        // it, 735 / 915)
        f32x4 y[ST];
        float top = 0.f;
#pragma unroll
        for (int t = 0; t < ST; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float u = s[t][e] * a.scale_over_cap;
            y[t][e] = s[t][e] * a.scale_log2 * tanh_over(u);
            top = fmaxf(top, fabsf(u));
          }
        if (__any(top > kCapSmall)) {
#pragma unroll
          for (int t = 0; t < ST; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float u = s[t][e] * a.scale_over_cap;
              const float z = a.cap_log2 * tanh_of<T>(u);
              y[t][e] = fabsf(u) > kCapSmall ? z : y[t][e];
            }
        }
#pragma unroll
        for (int t = 0; t < ST; ++t) s[t] = y[t];
      } else {
#pragma unroll
        for (int t = 0; t < ST; ++t) s[t] *= a.scale_log2;
      }
      const int4 w = info[(rg * NQ + n) * 16 + (lane & 15)];
      const int k1 = w.z - k0 - 4 * (lane >> 4);
#pragma unroll
      for (int t = 0; t < ST; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[t][e] -= __int_as_float(w.w) * fabsf((float)(k1 - (t * 16 + e)));
    };
    // probabilities of row block n against its reference, packed, what that
    // leaves over (FINE), and their sum; all: every row sees every key
    auto probs = [&](auto all, const f32x4 (&s)[ST], float ref, frag (&pf)[PF], frag (&pl)[PL]) {
      float ts = 0.f;
#pragma unroll
      for (int f = 0; f < PF; ++f) {
        float pv[KPL];
#pragma unroll
        for (int e = 0; e < KPL; ++e)
          pv[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[f * (KPL / 4) + e / 4][e % 4], cc, -ref));
        if constexpr (FINE) {
          // cut off, not rounded, so that the rest has the probability's sign; and
          // no rest of 0 where a value may be infinite (2^-126, the least that the
          // exponential returns)
          u32x4 top;
          float rest[KPL];
#pragma unroll
          for (int e = 0; e < KPL; ++e) {
            const uint32_t w = __float_as_uint(pv[e]);
            top[e / 2] = e % 2 ? top[e / 2] | (w & 0xffff0000u) : w >> 16;
            rest[e] = pv[e] - __uint_as_float(w & 0xffff0000u);
            if (decltype(all)::value) rest[e] = fmaxf(rest[e], 0x1p-126f);
            ts += pv[e];
          }
          pf[f] = __builtin_bit_cast(frag, top);
          pl[f] = pack_frag(rest, (frag*)nullptr);
        } else {
          pf[f] = pack_frag(pv, (frag*)nullptr);
          ts = frag_sum(pf[f], ts);
        }
      }
      return ts;
    };
    // The reference of a row is not its running maximum: it stays where it is
    // while a tile's probabilities sum to at most 2^24 (softmax does not depend
    // on it, and o and l stay far inside fp32), so most tiles need no maximum.
    // Rows that need it take the exact maximum of this tile, all four lanes of a
    // row alike; no row's rounding depends on another row.
    auto new_reference = [&](const f32x4 (&s)[ST], int n, bool raise) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < ST; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
      mx = row_max(mx) * cc;
      const float mn = raise ? fmaxf(m[n], mx) : m[n];
      // (nothing to scale before the first key; -inf - -inf is avoided)
      const float alpha = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - mn);
      l[n] *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) oacc[n][d] *= alpha;
      m[n] = mn;
    };
    auto reference = [&](int n) { return m[n] == -INFINITY ? 0.f : m[n]; };
    auto any_in_row = [&](bool x) {      // over the four lanes of a row
      const auto v = __builtin_amdgcn_permlane16_swap((unsigned)x, (unsigned)x, false, false);
      return halves_or((int)(v[0] | v[1])) != 0;
    };

    // S^T of KS keys: sub-tile t, row block n: keys 16 t + 4 g + [0, 4) of row c16
    auto scores = [&](const char* kt, int lane, f32x4 (&s)[NQ][ST]) {
#pragma unroll
      for (int t = 0; t < ST; ++t) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < QF; ++kk) {
          const frag kf = key_frag(kt, t, kk, lane);
#pragma unroll
          for (int n = 0; n < NQ; ++n) s[n][t] = MM::mma(kf, qf[n][kk], s[n][t]);
        }
      }
    };
    // KS keys that every row of the wave sees
    auto whole = [&](auto other, const char* kt, const char* vt, int k0) {
      f32x4 s[NQ][ST];
      scores(kt, lane, s);
      if constexpr (decltype(other)::value) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) transform(s[n], n, k0, lane);
      }
      // the first V fragments on their way before the scores are weighed (as many
      // as the registers hold without spilling; 8,192 queries over 12,288 keys
      // 1,220 us without, 1,150 with three or four)
      frag ve[PF][VE ? VE : 1];
#pragma unroll
      for (int f = 0; f < PF; ++f)
#pragma unroll
        for (int d = 0; d < VE; ++d) ve[f][d] = VO::template load<RB>(vt, f * VO::KEYS, d * 16, lane);
      if (VE) __builtin_amdgcn_sched_barrier(0);
      frag pf[NQ][PF], pl[NQ][PL];
      float ts[NQ];
      bool over[NQ], any = false;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        ts[n] = probs(std::true_type{}, s[n], reference(n), pf[n], pl[n]);
        over[n] = m[n] == -INFINITY || !(ts[n] <= kMostSum);
        any = any || over[n];
      }
      if (__any(any)) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          new_reference(s[n], n, any_in_row(over[n]));
          ts[n] = probs(std::true_type{}, s[n], reference(n), pf[n], pl[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) l[n] += ts[n];
      // this product ahead of the other wave's instructions, which then weighs its
      // scores under it: 1,117 / 1,091 us for 8,192 queries over 12,288 keys, fp32
      // and wide heads 3 to 8% (around the scores' product instead it costs 2%)
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int f = 0; f < PF; ++f)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const frag vf = d < VE ? ve[f][d < VE ? d : 0]
                                 : VO::template load<RB>(vt, f * VO::KEYS, d * 16, lane);
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            if constexpr (FINE) oacc[n][d] = MM::mma(vf, pl[n][f], oacc[n][d]);
            oacc[n][d] = MM::mma(vf, pf[n][f], oacc[n][d]);
          }
        }
      __builtin_amdgcn_s_setprio(0);
    };

    // Any other KS keys: keys that a row does not see, keys past the segment,
    // blocks that are none.
    auto masked = [&](const char* kt, const char* vt, int k0) {
      // (addresses formed anew in every call: kept from call to call they would
      // fill the registers that the loop over whole tiles needs)
      const int lane = lane_again();
      const int c16 = lane & 15, g = lane >> 4;
      f32x4 s[NQ][ST];
      scores(kt, lane, s);
      uint32_t see[NQ];            // visible bits of this lane's scores (bit t * 4 + e)
      frag pf[NQ][PF], pl[NQ][PL];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        if (general) transform(s[n], n, k0, lane);
        const int4 w = info[(rg * NQ + n) * 16 + c16];
        // of the lane's keys k0 + 4 g + 16 t + e, those in [lo, hi)
        const int lo = w.x - k0 - 4 * g, hi = min(w.y, seg_end) - k0 - 4 * g;
        see[n] = 0;
#pragma unroll
        for (int t = 0; t < ST; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            see[n] |= (t * 16 + e >= lo && t * 16 + e < hi) ? 1u << (t * 4 + e) : 0u;
        if (seg_bad) {
#pragma unroll 1
          for (int b = 0; b < ST * 4; ++b) {
            const int pg = (min(k0 + 4 * g + (b >> 2) * 16 + (b & 3), seg_end - 1) >> shift) - p0;
            if ((none[pg / 32] >> (pg % 32)) & 1) see[n] &= ~(1u << b);
          }
        }
#pragma unroll
        for (int t = 0; t < ST; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!((see[n] >> (t * 4 + e)) & 1)) s[n][t][e] = -INFINITY;
        float ts = probs(std::false_type{}, s[n], reference(n), pf[n], pl[n]);
        const bool over = m[n] == -INFINITY || !(ts <= kMostSum);
        if (__any(over)) {
          new_reference(s[n], n, any_in_row(over));
          ts = probs(std::false_type{}, s[n], reference(n), pf[n], pl[n]);
        }
        l[n] += ts;
      }
      // A value that is not finite must not reach a row that does not see its
      // key (0 * inf): such values are taken out, and added as what they do to
      // the rows that see them.
#pragma unroll
      for (int f = 0; f < PF; ++f)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          frag vf = VO::template load<RB>(vt, f * VO::KEYS, d * 16, lane);
          if (__any(VO::odd_bits(vf) != 0)) {
            const frag pos = VO::odd_part(vf, 0), neg = VO::odd_part(vf, 1);
            vf = VO::finite_part(vf);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
              float b[KPL];
#pragma unroll
              for (int e = 0; e < KPL; ++e) b[e] = (see[n] >> (f * KPL + e)) & 1 ? 1.f : 0.f;
              const frag one = pack_frag(b, (frag*)nullptr);
              const f32x4 zero{0.f, 0.f, 0.f, 0.f};
              const f32x4 cp = MM::mma(pos, one, zero), cn = MM::mma(neg, one, zero);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (cp[e] > 0.f) oacc[n][d][e] += INFINITY;
                if (cn[e] > 0.f) oacc[n][d][e] -= INFINITY;
              }
            }
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            if constexpr (FINE) oacc[n][d] = MM::mma(vf, pl[n][f], oacc[n][d]);
            oacc[n][d] = MM::mma(vf, pf[n][f], oacc[n][d]);
          }
        }
    };

    // ---- the segment's tiles: those before the window that every row of the
    // wave sees, those inside it, those after it.  Loops of their own, so that
    // the accumulators keep their registers through the one that counts; the
    // waves of a group may be in different ones, but each passes one barrier
    // per tile.
    auto first_key = [&](int i) { return seg + (i * KG + kg) * KT; };
    auto inside = [&](int i) {
      const int k0 = first_key(i);
      return !seg_bad && k0 >= wlo && k0 + KT <= min(whi, seg_end);
    };
    int i = 0, st = 0;
    auto turn = [&](auto&& work) {
      // every turn issues one tile (past the last one, a copy of it into a slot
      // nobody reads again), so tile i has landed once STAGES - 2 later ones
      // remain in flight
      wait_vmcnt<(STAGES - 2) * 2 * C::ROUNDS>();
      if (RG > 1) {   // ... in every wave's part, and the slot refilled below is idle
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
      if (i < mine) {
        issue(min(i + STAGES - 1, mine - 1), st == 0 ? STAGES - 1 : st - 1, lane);
        const char* kt = ring + st * 2 * C::TILE;
        if (!idle) work(kt, first_key(i));
      }
      st = st + 1 == STAGES ? 0 : st + 1;
      ++i;
    };
#pragma unroll
    for (int p = 0; p < STAGES - 1; ++p)
      if (mine > 0) issue(min(p, mine - 1), p, lane_again());
    auto whole_tile = [&](auto other) {
      return [&, other](const char* kt, int k0) {
#pragma unroll
        for (int h = 0; h < KT / KS; ++h)
          whole(other, kt + h * KS * RB, kt + C::TILE + h * KS * RB, k0 + h * KS);
      };
    };
    for (int pass = 0; pass < 2; ++pass) {
      while (i < iters && (pass == 1 || !inside(i)))
        turn([&](const char* kt, int k0) {
#pragma unroll 1
          for (int h = 0; h < KT / KS && k0 < seg_end; ++h, k0 += KS, kt += KS * RB)
            masked(kt, kt + C::TILE, k0);
        });
      if (general)
        while (i < iters && inside(i)) turn(whole_tile(std::true_type{}));
      else
        while (i < iters && inside(i)) turn(whole_tile(std::false_type{}));
    }
    wait_vmcnt<0>();
  }

  // ---- join the groups, write the result or the partial one
  float lt[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) lt[n] = row_sum(l[n]);
  const bool partial = a.always_partial || parts > 1;
  const int64_t prow = ((int64_t)slot * a.n_kv + head) * C::ROWS;
  if constexpr (KG == 1) {
    // (what depends on the lane or the group is formed anew, not kept in
    // registers till here)
    const int le = lane_again();
    int group = a.group;
    asm volatile("" : "+s"(group));
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int g = le >> 4, r = (rg * NQ + n) * 16 + (le & 15);
      if (r >= n_rows) continue;
      const float inv = lt[n] == 0.f ? 0.f : 1.f / lt[n];
      const int i = (row0 + r) / group, hd = head * group + row0 + r - i * group;
      const int64_t t = x.tok0 + i;
      T* op = static_cast<T*>(a.o) + t * a.o_token + (int64_t)hd * a.o_head;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        if (partial) {
          *reinterpret_cast<f32x4*>(a.part_o + (prow + r) * D + d * 16 + 4 * g) = oacc[n][d];
        } else {
          T w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = from_f32<T>(oacc[n][d][e] * inv);
          if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(op + d * 16 + 4 * g) = *reinterpret_cast<const uint2*>(w);
          else
            *reinterpret_cast<uint4*>(op + d * 16 + 4 * g) = *reinterpret_cast<const uint4*>(w);
        }
      }
      if (g == 0) {
        if (partial) a.part_ml[prow + r] = make_float2(m[n], lt[n]);
        else if (a.lse)
          a.lse[t * a.n_kv * a.group + hd] =
              lt[n] == 0.f ? -INFINITY : (m[n] + __log2f(lt[n])) / kLog2e;
      }
    }
  } else {
    // the groups' (max, sum, o) through LDS, then 8 dims of a row per thread
    float* mo = reinterpret_cast<float*>(lds);
    float2* ml = reinterpret_cast<float2*>(mo + KG * C::ROWS * C::MLD);
    __syncthreads();                       // every ring is idle
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int r = kg * C::ROWS + (rg * NQ + n) * 16 + c16;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<f32x4*>(mo + r * C::MLD + d * 16 + 4 * g) = oacc[n][d];
      if (g == 0) ml[r] = make_float2(m[n], lt[n]);
    }
    __syncthreads();
    const int per_row = D / 8;
    for (int idx = tid; idx < n_rows * per_row; idx += C::NT) {
      const int r = idx / per_row, d0 = (idx - r * per_row) * 8;
      float mx = -INFINITY, sum = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KG; ++k) mx = fmaxf(mx, ml[k * C::ROWS + r].x);
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int k = 0; k < KG; ++k) {
        const float2 w = ml[k * C::ROWS + r];
        if (w.y == 0.f) continue;          // saw nothing (a NaN sum counts)
        const float f = __builtin_amdgcn_exp2f((w.x == -INFINITY ? 0.f : w.x) - ref);
        sum += f * w.y;
        const float* x = mo + (k * C::ROWS + r) * C::MLD + d0;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += f * x[e];
      }
      if (partial) {
        float* po = a.part_o + (prow + r) * D + d0;
        *reinterpret_cast<f32x4*>(po) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(po + 4) = f32x4{v[4], v[5], v[6], v[7]};
        if (d0 == 0) a.part_ml[prow + r] = make_float2(mx, sum);
        continue;
      }
      const int i = (row0 + r) / a.group, hd = head * a.group + row0 + r - i * a.group;
      const int64_t t = x.tok0 + i;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= inv;
      Vec8<T> o8;
      o8.from_float(v);
      o8.store(static_cast<T*>(a.o) + t * a.o_token + (int64_t)hd * a.o_head + d0);
      if (d0 == 0 && a.lse)
        a.lse[t * a.n_kv * a.group + hd] = sum == 0.f ? -INFINITY : (mx + __log2f(sum)) / kLog2e;
    }
  }
}

// ------------------------------------------------------------------- merge
// Joins a row's partial results, those of the pass over the shared keys (pre)
// and those of its own unit: o = sum_j 2^(m_j - m) o_j / sum_j 2^(m_j - m) l_j.
// A workgroup takes RPW rows of one unit and KV head; 256 / RPW threads share
// a row, 4 dims each, the others taking every (STREAMS)-th part.  The weights
// go through LDS first, so that the loads of o depend on nothing.
constexpr int kMergeParts = 512;   // weights held at a time
template <typename T, int RPW>
__global__ __launch_bounds__(256) void attend_merge_kernel(AttendArgs a, SharedParts pre,
                                                           SeqTable tab, int row_blocks) {
  __shared__ float wts[RPW][kMergeParts / RPW];
  __shared__ __align__(16) float sums[256 * 4];
  __shared__ float lsum[256];
  constexpr int TPR = 256 / RPW, CHUNK = kMergeParts / RPW;
  const int D = a.head_dim, tpd = D / 4;                  // threads per part
  const int rb = blockIdx.x % row_blocks;
  const int head = blockIdx.x / row_blocks % a.n_kv, unit = blockIdx.x / row_blocks / a.n_kv;
  const Unit x = unit_of(a, tab, unit);
  const int row0 = x.tile * a.rows, n_rows = min(a.rows, x.nq * a.group - row0);
  if (rb * RPW >= n_rows) return;
  const int2 it = a.unit_items[unit];                     // first item, parts
  if (it.y == 1 && !a.always_partial) return;             // written already
  const int rl = threadIdx.x / TPR, tr = threadIdx.x % TPR;
  const int r = rb * RPW + rl;
  const bool valid = r < n_rows;
  const int rr = valid ? r : n_rows - 1;                  // (a row of its own for every thread)
  const int i = (row0 + rr) / a.group, g = row0 + rr - i * a.group;
  const int t = x.tok0 + i, h = head * a.group + g;
  const int n_pre = pre.splits, P = n_pre + it.y;
  // part j: row index into the partial results of its pass
  const int prow = t * a.group + g, ptile = n_pre ? prow / pre.rows : 0;
  const int64_t pre_at = ((int64_t)ptile * n_pre * a.n_kv + head) * pre.rows + prow - ptile * pre.rows;
  const int64_t own_at = ((int64_t)it.x * a.n_kv + head) * a.rows + rr;
  const int64_t pre_step = (int64_t)a.n_kv * pre.rows, own_step = (int64_t)a.n_kv * a.rows;
  auto ml_of = [&](int j) {
    return j < n_pre ? pre.part_ml[pre_at + j * pre_step] : a.part_ml[own_at + (j - n_pre) * own_step];
  };
  auto o_of = [&](int j) {
    return j < n_pre ? pre.part_o + (pre_at + j * pre_step) * D
                     : a.part_o + (own_at + (j - n_pre) * own_step) * D;
  };
  const int streams = TPR / tpd, sj = tr / tpd, d0 = (tr - sj * tpd) * 4;
  const bool active = sj < streams;
  // what the first parts left is on its way while their weights are found
  constexpr int EARLY = 8;
  const float2 none = make_float2(-INFINITY, 0.f);
  const float2 v0 = tr < P ? ml_of(tr) : none;
  f32x4 early[EARLY];
#pragma unroll
  for (int k = 0; k < EARLY; ++k) {
    const int j = sj + k * streams;
    early[k] = active && j < min(P, CHUNK) ? *reinterpret_cast<const f32x4*>(o_of(j) + d0)
                                           : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // maximum over the row's parts (a part that saw nothing has sum 0; a NaN sum
  // counts, its maximum may be -inf)
  float m = v0.y != 0.f ? v0.x : -INFINITY;
  for (int j = tr + TPR; j < P; j += TPR) {
    const float2 v = ml_of(j);
    if (v.y != 0.f) m = fmaxf(m, v.x);
  }
  constexpr int SH = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = SH / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (TPR > 64) {
    if ((threadIdx.x & 63) == 0) lsum[threadIdx.x / 64] = m;
    __syncthreads();
    m = fmaxf(fmaxf(lsum[0], lsum[1]), fmaxf(lsum[2], lsum[3]));
  }
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < P; j0 += CHUNK) {
    const int n = min(CHUNK, P - j0);
    __syncthreads();
    for (int j = tr; j < n; j += TPR) {
      const float2 v = j0 + j == tr ? v0 : ml_of(j0 + j);
      const float w = v.y == 0.f ? 0.f
                                 : __builtin_amdgcn_exp2f((v.x == -INFINITY ? 0.f : v.x) - ref);
      wts[rl][j] = w;
      l += w * v.y;
    }
    __syncthreads();
    if (active) {
      int j = sj;
      if (j0 == 0) {
#pragma unroll
        for (int k = 0; k < EARLY; ++k)
          if (sj + k * streams < n) o += wts[rl][sj + k * streams] * early[k];
        j = sj + EARLY * streams;
      }
#pragma unroll 8
      for (; j < n; j += streams)
        o += wts[rl][j] * *reinterpret_cast<const f32x4*>(o_of(j0 + j) + d0);
    }
  }
  // sums over the row's threads, in a fixed order
  *reinterpret_cast<f32x4*>(sums + threadIdx.x * 4) = o;
#pragma unroll
  for (int k = SH / 2; k > 0; k >>= 1) l += __shfl_xor(l, k);
  lsum[threadIdx.x] = l;
  __syncthreads();
  if (TPR > 64) l = (lsum[0] + lsum[64]) + (lsum[128] + lsum[192]);
  if (!valid || sj != 0) return;
  for (int k = 1; k < streams; ++k)
    o += *reinterpret_cast<const f32x4*>(sums + (threadIdx.x + k * tpd) * 4);
  T* op = static_cast<T*>(a.o) + (int64_t)t * a.o_token + (int64_t)h * a.o_head + d0;
  T w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = from_f32<T>(l == 0.f ? 0.f : o[e] / l);
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(op) = *reinterpret_cast<const uint2*>(w);
  else
    *reinterpret_cast<uint4*>(op) = *reinterpret_cast<const uint4*>(w);
  if (d0 == 0 && a.lse)
    a.lse[(int64_t)t * a.n_kv * a.group + h] =
        l == 0.f ? -INFINITY : (m + __log2f(l)) / kLog2e;
}

template <typename T>
hipError_t attend_merge(const AttendArgs& a, const SharedParts& pre, const SeqTable& tab,
                        int most_rows, hipStream_t s) {
  const int rows = most_rows < a.rows ? most_rows : a.rows;
  const int64_t tiles = (int64_t)a.n_units * a.n_kv;
  const int rpw = merge_rows(tiles, rows, a.head_dim), blocks = (rows + rpw - 1) / rpw;
  const int64_t groups = merge_groups(tiles, rows, a.head_dim);
  if (!fits_launch(groups, 256)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)groups);
  if (rpw == 1) {
    CR_LAUNCH((attend_merge_kernel<T, 1>), grid, dim3(256), 0, s, a, pre, tab, blocks);
  } else if (rpw == 8) {
    CR_LAUNCH((attend_merge_kernel<T, 8>), grid, dim3(256), 0, s, a, pre, tab, blocks);
  } else {
    CR_LAUNCH((attend_merge_kernel<T, 4>), grid, dim3(256), 0, s, a, pre, tab, blocks);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ launch
template <typename T, int D>
hipError_t attend_as(const AttendArgs& a, const SeqTable& tab, int64_t items, hipStream_t s) {
  const dim3 grid((unsigned)attend_groups(items, a.n_kv));
  constexpr int WIDE = attend_rows(sizeof(T), D), KEYS = ValueOps<T>::KEYS;
  constexpr int RB = tile_row_bytes(D * (int)sizeof(T));
  constexpr int OCC = attend_resident(sizeof(T), D);
  // 16 rows (the heads of a group for one new token): bound by reading the
  // keys.  Two waves with a ring of two 8 KB tiles of K and of V each (16 KB for
  // wide heads), two workgroups to a CU.
  constexpr int KN = 8192 / RB < KEYS ? KEYS : 8192 / RB;
  // wide units: a transfer of 1 KB for each of the four waves at least
  constexpr int KM = sizeof(T) == 2 && D <= 128 ? 2 * KEYS : KEYS;
  constexpr int KW = KM < 4096 / RB ? 4096 / RB : KM;
  if (a.rows == 16) {
    CR_LAUNCH((attend_kernel<T, D, 1, 1, 2, KN, 2>), grid, dim3(attend_threads(16)), 0, s, a, tab);
  } else if (a.rows == WIDE) {
    CR_LAUNCH((attend_kernel<T, D, WIDE / 64, 4, 1, KW, 2, OCC>), grid, dim3(attend_threads(WIDE)), 0,
              s, a, tab);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <typename T>
hipError_t attend(const AttendArgs& a, const SeqTable& tab, hipStream_t s) {
  const int64_t items = a.shared ? (int64_t)a.n_units * a.splits
                                 : (int64_t)a.n_units + (a.slots ? a.slots : 0);
  if (!fits_launch(attend_groups(items, a.n_kv), attend_threads(a.rows))) return hipErrorInvalidValue;
  switch (a.head_dim) {
    case 32: return attend_as<T, 32>(a, tab, items, s);
    case 64: return attend_as<T, 64>(a, tab, items, s);
    case 96: return attend_as<T, 96>(a, tab, items, s);
    case 128: return attend_as<T, 128>(a, tab, items, s);
    case 160: return attend_as<T, 160>(a, tab, items, s);
    case 192: return attend_as<T, 192>(a, tab, items, s);
    case 224: return attend_as<T, 224>(a, tab, items, s);
    case 256: return attend_as<T, 256>(a, tab, items, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace cr
