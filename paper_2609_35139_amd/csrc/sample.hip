// A token for every row of logits by temperature, top-k, top-p and min-p and a
// given random number (gfx950).
//
// Tokens stand in the order of their logits x, the lowest index of equal ones
// first (NaN counts as -inf, and -inf is never drawn).  With x_0 the largest,
//   p_i = exp((x_i - x_0) / T)
// and of the first k tokens (top-k) those stay for which the p before them sum
// to less than top_p times the sum over the k, and p_i >= min_p; the first one
// always.  The token is the first one, by index, up to which the p that stay
// sum to more than u times their sum.
//
// p is held as a whole number of 2^-44 (2^-42 for rows of more than 2^18
// logits): sums of whole numbers do not depend on their order, so every pass may
// add in the order that suits it, and what is off is the rounding of each p,
// 2^-45, a few 2^-36 of a sum of 2^18 of them.
#include <algorithm>
#include <type_traits>

#include "answer.h"
#include "sample_weights.h"

namespace cr {

constexpr int kSampleThreads = 512, kSampleWaves = kSampleThreads / 64;
constexpr int kSampleBins = 2048;
constexpr int kSampleList = 2048;     // tokens that are looked at one by one
// top-k that a list is made for at once (256 of 151,936: 35 us, by bins 55; 500: 77 and 56)
constexpr int kMostTopK = 256;
// of a list that is compared each with each (a row with top-k 20: 22 us, by bins 27; 100:
// 30 and 33; 200: 39 and 35)
constexpr int kSampleShort = 160;

typedef u64 Pair __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t order_of(float x) {      // whole numbers in the order of x
  const uint32_t b = __float_as_uint(x + 0.f);               // (-0 is 0)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// Where the tokens that stay end: those above v, and of those equal to v the ones
// up to index `last`.
struct Cut {
  float v = -INFINITY;
  int last = -1;
  __device__ __forceinline__ bool keeps(float x, int i) const {
    return (x > v) | ((x == v) & (i <= last));     // (no branches)
  }
};

struct SampleShared {
  u64 mass[kSampleBins];                // or sums of the row's chunks
  uint32_t count[kSampleBins];
  alignas(16) u64 list[kSampleList], few[kSampleList], weight[kSampleShort];
  double table[kExpTable];
  u64 scan[kSampleWaves];
  u64 word[4];
  uint32_t n_list, n_few;
  float range[2 * kSampleWaves];
};

// A row is read in chunks of U vectors for each lane of a wave, wave w taking chunks
// w, w + 8, ...: eight where a pass only compares (its loads are what it waits for: 7 us
// for 151,936 logits), four where it sums weights, one where it bins them (four: 3% slower,
// the bins' code is the longer).  What is done for a logit stands in
// the code once, for a vector or for four: a workgroup runs through most of this code
// once, and a line of it that is not in the instruction cache takes about a microsecond
// (everything unrolled over eight vectors: 180 KB, and 45 us for a pass that finds 360
// tokens; 9 to 13 now).
constexpr int kRead = 4, kReadMost = 2 * kRead;

template <typename T>
struct Sampler {
  static constexpr int NT = kSampleThreads, WAVES = kSampleWaves, VEC = 16 / sizeof(T);
  template <int U> static constexpr int CHUNK = 64 * VEC * U;
  SampleShared& sh;
  const T* row;
  int vocab;
  Weigher weigh;
  int tid, lane, wave;

  template <int U>
  __device__ __forceinline__ int chunks() const { return (vocab + CHUNK<U> - 1) / CHUNK<U>; }
  __device__ __forceinline__ static void elements(const uint4& w, float (&x)[VEC]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if constexpr (sizeof(T) == 2)
        x[e] = __uint_as_float(e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
      else
        x[e] = __uint_as_float(u[e]);
    }
  }
  // index of the first element of the lane's vector u of chunk c: vectors that pass
  // the end of the row are read from its last elements, those of them that another
  // vector holds as -inf
  template <int U>
  __device__ __forceinline__ int first_of(int c, int u) const {
    return min(c * CHUNK<U> + (u * 64 + lane) * VEC, vocab - VEC);
  }
  template <int U>
  __device__ __forceinline__ void load(int c, uint4 (&w)[U]) const {
    if (vocab >= VEC) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        __builtin_memcpy(&w[u], row + first_of<U>(c, u), 16);     // (rows begin anywhere)
      return;
    }
    // a row shorter than a vector, element by element
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int i = first_of<U>(c, u) + e;
        if (i < 0) continue;
        if constexpr (sizeof(T) == 2)
          v[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[i] << (e % 2 * 16);
        else
          v[e] = reinterpret_cast<const uint32_t*>(row)[i];
      }
      w[u] = uint4{v[0], v[1], v[2], v[3]};
    }
  }
  // ... and -inf in the places of elements that another vector holds
  template <int U>
  __device__ __forceinline__ void clear(int c, uint4 (&w)[U]) const {
    if ((c + 1) * CHUNK<U> <= vocab) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t v[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
      const int gone = c * CHUNK<U> + (u * 64 + lane) * VEC - first_of<U>(c, u);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (e >= gone) continue;
        if constexpr (sizeof(T) == 2)
          v[e / 2] = e % 2 ? (v[e / 2] & 0xffffu) | 0xff800000u : (v[e / 2] & 0xffff0000u) | 0xff80u;
        else
          v[e] = 0xff800000u;
      }
      w[u] = uint4{v[0], v[1], v[2], v[3]};
    }
  }
  // f(chunk, its vectors) for this wave's chunks, the next one on its way meanwhile
  template <int U, typename F>
  __device__ __forceinline__ void each_chunk(F&& f) const {
    const int n = chunks<U>();
    if (wave >= n) return;
    uint4 w[U], next[U];
    load<U>(wave, w);
#pragma unroll 1
    for (int c = wave; c < n; c += WAVES) {
      load<U>(min(c + WAVES, n - 1), next);
      clear<U>(c, w);
      f(c, w);
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = next[u];
    }
  }
  // f(vector number, its logits, the first one's index) for this wave's vectors, 64 lanes'
  // at a time: the code stands once, the loads are as far ahead as in each_chunk.
  template <typename F>
  __device__ __forceinline__ void each_vector(F&& f) const {
    each_chunk<kRead>([&](int c, uint4 (&w)[kRead]) {
#pragma unroll 1
      for (int u = 0; u < kRead; ++u) {
        float x[VEC];
        elements(w[0], x);
        f(c * kRead + u, x, first_of<kRead>(c, u));
#pragma unroll
        for (int i = 0; i + 1 < kRead; ++i) w[i] = w[i + 1];
      }
    });
  }
  // A bit for each of a vector's logits that the cut keeps, and all bits where bit e is set
  __device__ __forceinline__ static uint32_t kept_bits(const float (&x)[VEC], int i, const Cut& cut) {
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) bits |= (uint32_t)(x[e] > cut.v) << e;
    if (cut.last >= 0) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) bits |= (uint32_t)((x[e] == cut.v) & (i + e <= cut.last)) << e;
    }
    return bits;
  }
  __device__ __forceinline__ static u64 when_bit(uint32_t bits, int e) {
    return (u64)(int64_t)((int32_t)(bits << (31 - e)) >> 31);
  }
  // f(x, index) for the logits in [lo, hi] that `within` keeps: a bit for each of a
  // lane's logits, then the lanes' bits one after the other.
  template <typename F>
  __device__ __forceinline__ void each_of(float lo, float hi, const Cut& within, F&& f) const {
    each_chunk<kRead>([&](int c, const uint4 (&w)[kRead]) {
      bool any = false;
#pragma unroll
      for (int u = 0; u < kRead; ++u) {
        float x[VEC];
        elements(w[u], x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) any |= x[e] >= lo;
      }
      if (!__any(any)) return;
      uint32_t bits = 0;
#pragma unroll
      for (int u = 0; u < kRead; ++u) {
        float x[VEC];
        elements(w[u], x);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          bits |= (uint32_t)((x[e] >= lo) & (x[e] <= hi)) << (u * VEC + e);
      }
#pragma unroll 1
      while (__any(bits != 0)) {
        const int b = bits ? __ffs(bits) - 1 : 0;
        uint32_t v = 0;
#pragma unroll
        for (int d = 0; d < kRead * 4; ++d) {
          const uint4& four = w[d / 4];
          const uint32_t o = d % 4 == 0 ? four.x : d % 4 == 1 ? four.y : d % 4 == 2 ? four.z : four.w;
          v = b * (int)sizeof(T) / 4 == d ? o : v;
        }
        if constexpr (sizeof(T) == 2) v = b % 2 ? v & 0xffff0000u : v << 16;
        const float x = __uint_as_float(v);
        const int i = first_of<kRead>(c, b / VEC) + b % VEC;
        if (bits && within.keeps(x, i)) f(x, i);
        bits &= bits - 1;
      }
    });
  }
  // all bits, or none (selected by bits, a value is loaded whether it is needed or not,
  // and loads do not wait for each other's conditions)
  __device__ __forceinline__ static u64 when(bool c) { return 0 - (u64)c; }
  // (v of the lane that the data-parallel control names; 0 where there is none)
  template <int CTRL, int ROWS = 0xf>
  __device__ __forceinline__ static u64 lane_of(u64 v) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
    return (u64)hi << 32 | lo;
  }
  // sum over the lanes up to this one within 16, then within the wave
  __device__ __forceinline__ static u64 row_upto(u64 v) {
    v += lane_of<0x111>(v);               // row_shr:1, 2, 4, 8
    v += lane_of<0x112>(v);
    v += lane_of<0x114>(v);
    v += lane_of<0x118>(v);
    return v;
  }
  __device__ __forceinline__ static u64 wave_upto(u64 v) {
    v = row_upto(v);
    v += lane_of<0x142, 0xa>(v);          // row_bcast:15 into rows 1 and 3
    v += lane_of<0x143, 0xc>(v);          // row_bcast:31 into rows 2 and 3
    return v;
  }
  __device__ __forceinline__ static u64 at_lane(u64 v, int l) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
  }
  // sum of v over the threads before this one, and over all
  __device__ __forceinline__ u64 before(u64 v, u64* total) const {
    static_assert(WAVES <= 16, "a row of lanes");
    const u64 upto = wave_upto(v);
    __syncthreads();
    if (lane == 63) sh.scan[wave] = upto;
    __syncthreads();
    const u64 w = row_upto(lane < WAVES ? sh.scan[lane] : 0);
    *total = at_lane(w, WAVES - 1);
    return upto - v + (wave > 0 ? at_lane(w, wave - 1) : 0);
  }
  __device__ __forceinline__ u64 all(u64 v) const {
    u64 t;
    before(v, &t);
    return t;
  }
  __device__ __forceinline__ static u64 entry(float x, int i) {
    return (u64)order_of(x) << 32 | (0xffffffffu - (uint32_t)i);
  }
  __device__ __forceinline__ static float entry_value(u64 e) { return value_of((uint32_t)(e >> 32)); }
  __device__ __forceinline__ static int entry_index(u64 e) { return (int)(0xffffffffu - (uint32_t)e); }
  // the tokens in [lo, hi] that `within` keeps and f accepts, in the list; more than it
  // holds are only counted
  template <typename F>
  __device__ __forceinline__ uint32_t collect(float lo, float hi, const Cut& within, F&& f) const {
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    each_of(lo, hi, within, [&](float x, int i) {
      if (!f(x)) return;
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < (uint32_t)kSampleList) sh.list[at] = entry(x, i);
    });
    __syncthreads();
    return sh.n_list;
  }
  // ---- bins: of values from hi down, in `count` and (weights) `mass`
  // (in 64 bits: no difference of two logits overflows or vanishes)
  __device__ __forceinline__ static int bin_of(float x, float hi, double scale) {
    return min(kSampleBins - 1, (int)(((double)hi - (double)x) * scale));
  }
  __device__ __forceinline__ static double scale_of(float lo, float hi) {
    return hi > lo ? (double)(kSampleBins - 1) / ((double)hi - (double)lo) : 0.;
  }
  // the values that bins from `first` to `last` may hold
  __device__ __forceinline__ static float2 values_of(int first, int last, float lo, float hi, double scale) {
    if (!(scale > 0.)) return float2{lo, hi};
    return float2{fmaxf(lo, (float)((double)hi - (double)(last + 2) / scale)),
                  first > 0 ? (float)((double)hi - (double)(first - 1) / scale) : hi};
  }
  __device__ __forceinline__ void clear_bins() const {
    __syncthreads();
    for (int i = tid; i < kSampleBins; i += NT) { sh.mass[i] = 0; sh.count[i] = 0; }
    __syncthreads();
  }
  // The bin in which the running sum (of tokens, or of weight), from `above` on, reaches
  // `need`; what stands before it; the tokens up to its end.  bin kSampleBins: none does.
  struct Found { int bin; u64 above; uint32_t tokens; };
  __device__ __forceinline__ Found find(bool by_weight, u64 need, u64 above) const {
    constexpr int PER = kSampleBins / NT;
    __syncthreads();
    u64 c[PER], mine = 0, total;
    uint32_t tokens = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint32_t n = sh.count[tid * PER + i];
      c[i] = by_weight ? sh.mass[tid * PER + i] : n;
      mine += c[i];
      tokens += n;
    }
    u64 at = above + before(mine, &total), all;
    uint32_t upto = (uint32_t)before(tokens, &all);
    if (tid == 0) sh.word[0] = kSampleBins;
    __syncthreads();
    if (at < need && at + mine >= need) {
      bool found = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (found) continue;
        upto += sh.count[tid * PER + i];
        found = at + c[i] >= need;
        if (found) sh.word[0] = tid * PER + i;
        else at += c[i];
      }
      sh.word[1] = at;
      sh.word[2] = upto;
    }
    __syncthreads();
    return Found{(int)sh.word[0], sh.word[1], (uint32_t)sh.word[2]};
  }
  // Of the n entries of `few`, the one up to which, in descending order and from `above`
  // on, the sum reaches `need` (the last one if none does).
  __device__ __forceinline__ u64 pick(bool by_weight, int n, u64 need, u64 above) const {
    __syncthreads();
    // (their weights lie in `mass`: the bins have been looked at)
    for (int p = tid; p < n; p += NT) sh.mass[p] = by_weight ? weigh(entry_value(sh.few[p])) : 1;
    __syncthreads();
    for (int p = tid; p < n; p += NT) {
      const u64 e = sh.few[p];
      u64 b = above;
      bool last = true;
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const u64 o = sh.few[i];
        b += sh.mass[i] & when(o > e);
        last &= o >= e;
      }
      const u64 w = sh.mass[p];
      if (b < need && (b + w >= need || last)) sh.word[3] = e;
    }
    __syncthreads();
    return sh.word[3];
  }

  // The bins of [lo, hi] of the tokens that `within` keeps; returns the weight of all of
  // those, of any value, where by_weight.  Tokens that are few among the row's (and only
  // counted) are looked for first: 23 us instead of 38 for one in 50 of 151,936, but 71
  // for one in 3.
  __device__ __forceinline__ u64 bins(bool by_weight, bool few, float lo, float hi, const Cut& within) const {
    const double scale = scale_of(lo, hi);
    clear_bins();
    u64 sum = 0;
    if (few && !by_weight) {
      each_of(lo, hi, within, [&](float x, int) { atomicAdd(&sh.count[bin_of(x, hi, scale)], 1u); });
      __syncthreads();
      return 0;
    }
    auto dense = [&](auto weighed) {
      each_chunk<1>([&](int c, const uint4 (&w)[1]) {
        float x[VEC];
        u64 q[VEC];
        elements(w[0], x);
        const int i = first_of<1>(c, 0);
        if constexpr (weighed) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) q[e] = weigh(x[e]);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const bool kept = within.keeps(x[e], i + e);
          if constexpr (weighed) sum += q[e] & when(kept);
          if (kept & (x[e] >= lo) & (x[e] <= hi)) {
            const int b = bin_of(x[e], hi, scale);
            atomicAdd(&sh.count[b], 1u);
            if constexpr (weighed) atomicAdd(&sh.mass[b], q[e]);
          }
        }
      });
    };
    if (by_weight) dense(std::true_type{});
    else dense(std::false_type{});
    return all(sum);
  }
  __device__ __forceinline__ void reduce_range(float& least, float& most) const {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      least = fminf(least, __shfl_xor(least, o));
      most = fmaxf(most, __shfl_xor(most, o));
    }
    __syncthreads();
    if (lane == 0) { sh.range[wave] = least; sh.range[kSampleWaves + wave] = most; }
    __syncthreads();
    least = sh.range[lane % kSampleWaves];
    most = sh.range[kSampleWaves + lane % kSampleWaves];
#pragma unroll
    for (int o = kSampleWaves / 2; o > 0; o >>= 1) {
      least = fminf(least, __shfl_xor(least, o));
      most = fmaxf(most, __shfl_xor(most, o));
    }
  }

  // ---- the row in order: the sum of f over every chunk, and the token up to which
  // f first sums to more than `target`, given those sums.  f(logits of a vector, index
  // of the first, their shares).
  template <typename F>
  __device__ __forceinline__ u64 sum_chunks(F&& f) const {
    __syncthreads();
    u64 mine = 0;
    each_vector([&](int v, const float (&x)[VEC], int i) {
      u64 q[VEC], t = 0;
      f(x, i, q);
#pragma unroll
      for (int e = 0; e < VEC; ++e) t += q[e];
      mine += t;
      t = wave_upto(t);
      if (lane == 63) sh.mass[v] = t;
    });
    return all(mine);
  }
  template <typename F>
  __device__ __forceinline__ int locate(u64 target, F&& f) const {
    static_assert(kMostVocab / (64 * VEC) <= kSampleBins, "sums");
    const int n = chunks<kRead>() * kRead, per = (n + NT - 1) / NT;
    u64 mine = 0, total;
    for (int i = tid * per; i < min(n, tid * per + per); ++i) mine += sh.mass[i];
    u64 at = before(mine, &total);
    if (at <= target && at + mine > target) {
      int i = tid * per;
      while (at + sh.mass[i] <= target) at += sh.mass[i++];
      sh.word[0] = i;
      sh.word[1] = at;
    }
    __syncthreads();
    if (wave == 0) {
      const int c = (int)sh.word[0], i = first_of<1>(c, 0);
      uint4 w[1];
      float x[VEC];
      u64 q[VEC], t = 0;
      load<1>(c, w);
      clear<1>(c, w);
      elements(w[0], x);
      f(x, i, q);
#pragma unroll
      for (int e = 0; e < VEC; ++e) t += q[e];
      const u64 incl = wave_upto(t);
      u64 b = sh.word[1] + incl - t;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (b <= target && b + q[e] > target) sh.word[2] = i + e;
        b += q[e];
      }
    }
    __syncthreads();
    const int r = (int)sh.word[2];
    __syncthreads();
    return r;
  }
  // the take-th token, by index, of those equal to v that `within` keeps
  __device__ __forceinline__ int index_of_equal(float v, u64 take, const Cut& within) const {
    auto one = [&](const float (&x)[VEC], int i, u64 (&q)[VEC]) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) q[e] = x[e] == v && within.keeps(x[e], i + e);
    };
    sum_chunks(one);
    return locate(take - 1, one);
  }
  // less than this stands before a token that top-p lets stay
  __device__ __forceinline__ static u64 share_of(float top_p, u64 total) {
    return (u64)ceil((double)top_p * (double)total);
  }
  __device__ __forceinline__ static u64 target_of(float u, u64 total) {
    const double t = (double)u * (double)total;
    return t > 0. ? min((u64)t, total - 1) : 0;
  }

  // ---- everything on a list of the first n tokens (all that may stay).  of: the weight
  // that top-p is a share of (0: that of the first k of the list).  Returns the entry
  // drawn.
  __device__ __forceinline__ u64 from_list(int n, u64 k, float top_p, float least, u64 of, float u,
                                           u64* kept_weight) const {
    return n <= kSampleShort ? from_short_list(n, k, top_p, least, of, u, kept_weight)
                             : from_long_list(n, k, top_p, least, of, u, kept_weight);
  }
  // each entry compared with each
  __device__ __forceinline__ u64 from_short_list(int n, u64 k, float top_p, float least, u64 of,
                                                 float u, u64* kept_weight) const {
    static_assert(kSampleList <= kSampleBins, "weights of `few`");
    static_assert(kSampleShort <= NT, "an entry for each thread");
    const bool mine = tid < n;
    const u64 e = mine ? sh.list[tid] : 0;
    u64 q = mine ? weigh(entry_value(e)) : 0;
    if (mine) sh.weight[tid] = q;
    if (tid == n && n % 2) sh.list[n] = sh.weight[n] = 0;
    __syncthreads();
    u64 b = 0;
    uint32_t rank = 0;
    if (mine) {
#pragma unroll 4
      for (int i = 0; i < n; i += 2) {           // (an entry of 0 behind an odd number)
        const Pair o = *reinterpret_cast<const Pair*>(sh.list + i), w = *reinterpret_cast<const Pair*>(sh.weight + i);
        b += (w[0] & when(o[0] > e)) + (w[1] & when(o[1] > e));
        rank += (o[0] > e) + (o[1] > e);
      }
    }
    const bool within = mine && (k == 0 || rank < k);
    if (of == 0) of = all(within ? q : 0);
    const u64 share = top_p < 1.f ? share_of(top_p, of) : ~0ull;
    const bool stays = within && (rank == 0 || (b < share && entry_value(e) >= least));
    q = stays ? q : 0;
    __syncthreads();
    if (mine) sh.weight[tid] = q;
    const u64 kept = all(q);
    const u64 target = target_of(u, kept);
    if (stays) {
      u64 at = 0;                          // of lower indexes: larger lower halves
#pragma unroll 4
      for (int i = 0; i < n; i += 2) {
        const Pair o = *reinterpret_cast<const Pair*>(sh.list + i), w = *reinterpret_cast<const Pair*>(sh.weight + i);
        at += (w[0] & when((uint32_t)o[0] > (uint32_t)e)) + (w[1] & when((uint32_t)o[1] > (uint32_t)e));
      }
      if (at <= target && at + q > target) sh.word[3] = e;
    }
    __syncthreads();
    *kept_weight = kept;
    return sh.word[3];
  }
  // by bins of the values, then by bins of the indexes
  __device__ __forceinline__ u64 from_long_list(int n, u64 k, float top_p, float least, u64 of,
                                                float u, u64* kept_weight) const {
    constexpr int PER = kSampleList / NT;
    u64 e[PER], q[PER];
    float lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      e[i] = tid + i * NT < n ? sh.list[tid + i * NT] : 0;
      const float x = entry_value(e[i]);
      q[i] = e[i] ? weigh(x) : 0;
      if (e[i]) { lo = fminf(lo, x); hi = fmaxf(hi, x); }
    }
    reduce_range(lo, hi);
    const double scale = scale_of(lo, hi);
    // the last entry that stays by `need`: those below it lose their weight
    auto cut_at = [&](bool by_weight, u64 need) {
      clear_bins();
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (e[i]) {
          const int b = bin_of(entry_value(e[i]), hi, scale);
          atomicAdd(&sh.count[b], 1u);
          atomicAdd(&sh.mass[b], q[i]);
        }
      if (tid == 0) sh.n_few = 0;
      const Found f = find(by_weight, need, 0);
      if (f.bin >= kSampleBins) return;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (e[i] && bin_of(entry_value(e[i]), hi, scale) == f.bin) sh.few[atomicAdd(&sh.n_few, 1u)] = e[i];
      __syncthreads();
      const u64 last = pick(by_weight, (int)sh.n_few, need, f.above);
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (e[i] < last) e[i] = q[i] = 0;
    };
    auto sum = [&] {
      u64 t = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) t += q[i];
      return all(t);
    };
    if (k > 0 && k < (u64)n) cut_at(false, k);
    if (top_p < 1.f) cut_at(true, share_of(top_p, of ? of : sum()));
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (e[i] && entry_value(e[i]) < least) e[i] = q[i] = 0;
    const u64 kept = sum();
    // bins of 2^s indexes
    const u64 target = target_of(u, kept);
    int s = 0;
    while (((vocab - 1) >> s) >= kSampleBins) ++s;
    clear_bins();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (e[i]) atomicAdd(&sh.mass[entry_index(e[i]) >> s], q[i]);
    if (tid == 0) sh.n_few = 0;
    const Found f = find(true, target + 1, 0);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (e[i] && (entry_index(e[i]) >> s) == f.bin) sh.few[atomicAdd(&sh.n_few, 1u)] = e[i];
    __syncthreads();
    // (of lower indexes: larger lower halves)
    const int m = (int)sh.n_few;
    for (int p = tid; p < m; p += NT) sh.mass[p] = weigh(entry_value(sh.few[p]));
    __syncthreads();
    for (int p = tid; p < m; p += NT) {
      const u64 o = sh.few[p];
      u64 at = f.above;
#pragma unroll 8
      for (int i = 0; i < m; ++i) at += sh.mass[i] & when((uint32_t)sh.few[i] > (uint32_t)o);
      if (at <= target && at + sh.mass[p] > target) sh.word[3] = o;
    }
    __syncthreads();
    *kept_weight = kept;
    return sh.word[3];
  }
};

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  using S = Sampler<T>;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
  const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
  const float min_p = a.min_ps ? a.min_ps[r] : a.min_p;
  const int k_in = a.top_ks ? a.top_ks[r] : a.top_k;
  const float u = a.u[r];
  S s{sh, static_cast<const T*>(a.logits) + (int64_t)r * a.stride, a.vocab, Weigher{}, tid, lane, wave};
  const int shift = a.vocab <= (1 << 18) ? 44 : 42;
  // (a NaN among the settings leaves the first token)
  const bool greedy = !(temperature > 0.f) || k_in == 1 || !(top_p > 0.f) || !(min_p <= 1.f);

  // ---- the largest logit, of each thread (and the chunk where it first stands) and of
  // all
  float mine = -INFINITY;
  int where = 0;
  s.template each_chunk<kReadMost>([&](int c, const uint4 (&w)[kReadMost]) {
    float most = mine;
#pragma unroll
    for (int v = 0; v < kReadMost; ++v) {
      float x[S::VEC];
      S::elements(w[v], x);
#pragma unroll
      for (int e = 0; e < S::VEC; ++e) most = x[e] > most ? x[e] : most;
    }
    where = most > mine ? c : where;
    mine = most;
  });
  float low = mine > -INFINITY ? mine : INFINITY, top = mine;
  s.reduce_range(low, top);
  auto answer = [&](int token, float log_p) {
    if (tid != 0) return;
    a.tokens[r] = token;
    if (a.log_probs) a.log_probs[r] = log_p;
  };
  if (top == -INFINITY) return answer(-1, -INFINITY);
  if (greedy) {
    int first = 0x7fffffff;
    if (mine == top) {
      uint4 w[kReadMost];
      s.template load<kReadMost>(where, w);
      s.template clear<kReadMost>(where, w);
#pragma unroll
      for (int v = kReadMost - 1; v >= 0; --v) {
        float x[S::VEC];
        S::elements(w[v], x);
#pragma unroll
        for (int e = S::VEC - 1; e >= 0; --e)
          if (x[e] == top) first = s.template first_of<kReadMost>(where, v) + e;
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o));
    __syncthreads();
    if (lane == 0) sh.count[wave] = (uint32_t)first;
    __syncthreads();
    for (int i = 0; i < kSampleWaves; ++i) first = min(first, (int)sh.count[i]);
    return answer(first, 0.f);
  }
  const u64 k = k_in <= 0 || k_in >= a.vocab ? 0 : (u64)k_in;
  const double c = kExpTable * 1.4426950408889634074 / (double)temperature, at_top = top * c;
  if (top == INFINITY || !(fabs(at_top) < 0x1p48)) {
    // infinite ones, or so far from 0 that any other logit is too far from them: all of
    // the same weight
    auto equal = [&](const float (&x)[S::VEC], int, u64 (&q)[S::VEC]) {
#pragma unroll
      for (int e = 0; e < S::VEC; ++e) q[e] = x[e] == top;
    };
    const u64 n = s.sum_chunks(equal);
    u64 m = k > 0 && k < n ? k : n;
    if (top_p < 1.f) m = S::share_of(top_p, m);
    return answer(s.locate(S::target_of(u, m), equal), -(float)log((double)m));
  }
  const double one = ldexp(1., shift);
  if (tid < kExpTable) sh.table[tid] = Weigher::entry(tid, top, c, one);
  s.weigh = Weigher::of(sh.table, top, c);
  // (the largest logit's own weight, which may be off by a step: alone, its log is 0)
  auto finish = [&](int token, float x, u64 total) {
    const double q = (double)s.weigh(top);
    answer(token, (float)(((double)x - (double)top) / (double)temperature - log((double)total / q)));
  };
  // no token below `least` can stay by min_p
  constexpr float kLowest = kLowestLogit;
  const float least = min_p > 0.f ? least_logit(min_p, top, temperature) : kLowest;
  __syncthreads();                         // (the table)

  // ---- the tokens that may stay, where they are few enough for the list: all of them,
  // those from the k-th largest of the threads' largest on (at least k tokens are not
  // below it), those from `least` on
  int n_list = -1;
  u64 of = 0;                              // the weight of all, where top-p needs it
  Cut cut;                                 // where those that stay end
  float bound = INFINITY;
  if (a.vocab <= kSampleList) {
    bound = kLowest;
  } else if (k > 0 && k <= (u64)kMostTopK) {
    const double scale = S::scale_of(low, top);
    s.clear_bins();
    const int bin = mine > -INFINITY ? S::bin_of(mine, top, scale) : kSampleBins;
    if (bin < kSampleBins) atomicAdd(&sh.count[bin], 1u);
    const auto f = s.find(false, k, 0);
    if (f.bin < kSampleBins) {
      float most = top;
      bound = bin <= f.bin ? mine : top;
      s.reduce_range(bound, most);
    }
  } else if (k == 0 && top_p >= 1.f && min_p > 0.f) {
    bound = least;
  }
  if (bound < INFINITY) {
    const uint32_t n = s.collect(bound, top, Cut{}, [](float) { return true; });
    if (n <= (uint32_t)kSampleList) n_list = (int)n;
  }
  // ---- else where the first k end, then where top-p ends: by bins of the values, from a
  // bound down to which they are likely to lie (about one in 50 tokens is not below the
  // least of the threads' largest), or below which hardly a token can stay (by their logits
  // all of them together weigh less than 1 - top_p; what is held of each may be up to half
  // a step more); if it lies lower it is looked for among all; the bin in which the end lies
  // becomes the range, until its tokens fit the list or are all equal
#pragma unroll 1
  for (int stage = 0; stage < 2; ++stage) {
    const bool by_weight = stage == 1;
    if (n_list >= 0 || (by_weight ? !(top_p < 1.f) : k == 0)) continue;
    const Cut within = cut;
    const bool few = k * 100 <= (u64)a.vocab;
    float lo = by_weight ? at_most(top + (double)temperature * (logf((1.f - top_p) / (float)a.vocab) - 0.01f))
                         : fmaxf(kLowest, few ? low : low - (top - low));
    float hi = top;
    u64 need = k, above = 0;
#pragma unroll 1
    for (bool first = true;; first = false) {
      const u64 sum = s.bins(by_weight, few, lo, hi, within);
      if (by_weight && first) {
        of = sum;
        need = S::share_of(top_p, of);
      }
      const auto f = s.find(by_weight, need, above);
      if (f.bin >= kSampleBins) {
        if (lo == kLowest) break;                      // all of them stay
        lo = kLowest;                                  // the end lies below the bound
        continue;
      }
      const double scale = S::scale_of(lo, hi);
      const bool whole = hi == top && f.tokens <= (uint32_t)kSampleList;   // all up to the end
      const uint32_t n = sh.count[f.bin];
      const float2 v = S::values_of(whole ? 0 : f.bin, f.bin, lo, hi, scale);
      if (whole || n <= (uint32_t)kSampleList) {
        const int from = whole ? 0 : f.bin;
        const uint32_t got = s.collect(v.x, v.y, within, [&](float x) {
          const int b = S::bin_of(x, hi, scale);
          return b >= from && b <= f.bin && x >= lo && x <= hi;
        });
        if (whole) {
          n_list = (int)got;
          break;
        }
        for (int p = tid; p < (int)n; p += S::NT) sh.few[p] = sh.list[p];
        const u64 e = s.pick(by_weight, (int)n, need, f.above);
        cut = Cut{S::entry_value(e), S::entry_index(e)};
        break;
      }
      float least_here = INFINITY, most_here = -INFINITY;
      s.each_of(v.x, v.y, within, [&](float x, int) {
        if (S::bin_of(x, hi, scale) == f.bin) {
          least_here = fminf(least_here, x);
          most_here = fmaxf(most_here, x);
        }
      });
      s.reduce_range(least_here, most_here);
      if (least_here == most_here) {
        // equal ones: the first of them, by index
        const u64 w = by_weight ? s.weigh(most_here) : 1;
        cut = Cut{most_here, s.index_of_equal(most_here, (need - f.above + w - 1) / w, within)};
        break;
      }
      lo = least_here;
      hi = most_here;
      above = f.above;
    }
  }
  u64 total;
  if (n_list >= 0) {
    const u64 e = s.from_list(n_list, k, top_p, least, of, u, &total);
    return finish(S::entry_index(e), S::entry_value(e), total);
  }
  // ---- many: their sums in order of the index
  if (least > cut.v) cut = Cut{nextafterf(least, -INFINITY), -1};
  auto weight = [&](const float (&x)[S::VEC], int i, u64 (&q)[S::VEC]) {
    const uint32_t kept = S::kept_bits(x, i, cut);
#pragma unroll
    for (int e = 0; e < S::VEC; ++e) q[e] = 0;
    if (!__any(kept != 0)) return;
#pragma unroll
    for (int e = 0; e < S::VEC; ++e) q[e] = s.weigh(x[e]) & S::when_bit(kept, e);
  };
  total = s.sum_chunks(weight);
  const int token = s.locate(S::target_of(u, total), weight);
  if (tid == 0) finish(token, to_f32(s.row[token]), total);
}

template <typename T>
hipError_t sample(const SampleArgs& a, hipStream_t s) {
  CR_LAUNCH((sample_kernel<T>), dim3(a.n_rows), dim3(kSampleThreads), 0, s, a);
  return hipGetLastError();
}
template hipError_t sample<bf16>(const SampleArgs&, hipStream_t);
template hipError_t sample<float>(const SampleArgs&, hipStream_t);

}  // namespace cr
