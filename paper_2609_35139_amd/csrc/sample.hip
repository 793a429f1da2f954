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

#include "answer.h"

namespace cr {

constexpr int kSampleThreads = 512, kSampleWaves = kSampleThreads / 64;
constexpr int kSampleBins = 2048;
constexpr int kSampleList = 2048;     // tokens that are sorted

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t order_of(float x) {      // whole numbers in the order of x
  const uint32_t b = __float_as_uint(x + 0.f);               // (-0 is 0)
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// exp(d / T) 2^shift for d = x - x_0 <= 0, by t = 256 log2(e) d / T = n + r:
// 2^(n / 256) from a table and the exponent, e^(r log 2 / 256) by its series up to
// the fourth power (relative error 4e-17).
struct Weigher {
  const double* table;   // 2^(j / 256) 2^shift
  double top, c;         // 256 log2(e) / T
  __device__ __forceinline__ double scaled(float x) const {
    const double t = ((double)x - top) * c;
    if (!(t >= -64. * 256.)) return 0.;
    const double kMagic = 6755399441055744.;                 // 1.5 2^52
    const double m = t + kMagic;
    const int n = (int)(__double_as_longlong(m) & 0xffffffff);
    const double y = (t - (m - kMagic)) * 0.0027076061740622863;   // log(2) / 256
    double e = __builtin_fma(y, 1. / 24., 1. / 6.);
    e = __builtin_fma(e, y, 0.5);
    e = __builtin_fma(e, y, 1.);
    e = __builtin_fma(e, y, 1.);
    const long long b = __double_as_longlong(table[n & 255]) + ((long long)(n >> 8) << 52);
    return __longlong_as_double(b) * e;
  }
  __device__ __forceinline__ static u64 whole(double v) {      // v < 2^52, rounded
    return (u64)__double_as_longlong(v + 4503599627370496.) & ((1ull << 52) - 1);
  }
  __device__ __forceinline__ u64 operator()(float x) const { return whole(scaled(x)); }
};

// Where the tokens that stay end: those above v, and of those equal to v the ones
// up to index `last`.
struct Cut {
  float v = -INFINITY;
  int last = -1;
  __device__ __forceinline__ bool keeps(float x, int i) const {
    return x > v || (x == v && i <= last);
  }
};

struct SampleShared {
  u64 mass[kSampleBins];
  uint32_t count[kSampleBins];
  u64 list[kSampleList], weight[kSampleList];
  u64 sums[kMostVocab / 256];       // of every wave's pieces of the row
  double table[256];
  u64 scan[kSampleWaves];
  u64 word[4];
  uint32_t n_list;
  float range[2 * kSampleWaves];
};

template <typename T>
struct Sampler {
  static constexpr int NT = kSampleThreads, VEC = 4;
  SampleShared& sh;
  const T* row;
  int vocab;
  bool vectors;          // the row begins on four logits
  bool infinite;         // the largest logit is infinite: it and its equals alone count
  Weigher weigh;
  int tid, lane, wave;

  __device__ __forceinline__ int pieces() const { return (vocab + NT * VEC - 1) / (NT * VEC); }
  __device__ __forceinline__ void load(int j, int thread, float (&x)[VEC]) const {
    const int i = (j * NT + thread) * VEC;
    if (vectors && i + VEC <= vocab) {
      if constexpr (sizeof(T) == 2) {
        const uint2 w = *reinterpret_cast<const uint2*>(row + i);
        x[0] = __uint_as_float(w.x << 16);
        x[1] = __uint_as_float(w.x & 0xffff0000u);
        x[2] = __uint_as_float(w.y << 16);
        x[3] = __uint_as_float(w.y & 0xffff0000u);
      } else {
        const float4 w = *reinterpret_cast<const float4*>(row + i);
        x[0] = w.x;
        x[1] = w.y;
        x[2] = w.z;
        x[3] = w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] = i + e < vocab ? to_f32(row[i + e]) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (!(x[e] > -INFINITY)) x[e] = -INFINITY;
      if (infinite) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
    }
  }
  // f(x, index) for this thread's logits above -inf
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int n = pieces();
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      float x[VEC];
      load(j, tid, x);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (x[e] > -INFINITY) f(x[e], (j * NT + tid) * VEC + e);
    }
  }
  // sum of v over the threads before this one, and over all
  __device__ __forceinline__ u64 before(u64 v, u64* total) {
    u64 x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const u64 y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) sh.scan[wave] = x;
    __syncthreads();
    u64 b = x - v, t = 0;
    for (int i = 0; i < kSampleWaves; ++i) {
      if (i < wave) b += sh.scan[i];
      t += sh.scan[i];
    }
    *total = t;
    return b;
  }
  __device__ __forceinline__ u64 all(u64 v) {
    u64 t;
    before(v, &t);
    return t;
  }
  // the n entries of the list in descending order
  __device__ __forceinline__ void sort(u64* list, int n) {
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) list[i] = 0;
    for (int k = 2; k <= size; k *= 2)
      for (int d = k / 2; d > 0; d /= 2) {
        __syncthreads();
        for (int p = tid; p < size / 2; p += NT) {
          const int i = ((p & ~(d - 1)) << 1) | (p & (d - 1));
          const u64 a = list[i], b = list[i + d];
          if ((a < b) == ((i & k) == 0)) { list[i] = b; list[i + d] = a; }
        }
      }
    __syncthreads();
  }
  __device__ __forceinline__ static u64 entry(float x, int i) {
    return (u64)order_of(x) << 32 | (0xffffffffu - (uint32_t)i);
  }
  __device__ __forceinline__ static float entry_value(u64 e) { return value_of((uint32_t)(e >> 32)); }
  __device__ __forceinline__ static int entry_index(u64 e) { return (int)(0xffffffffu - (uint32_t)e); }
  // tokens that f accepts, in the list; more than it holds are only counted
  template <typename F>
  __device__ __forceinline__ uint32_t collect(F&& f) {
    __syncthreads();
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    each([&](float x, int i) {
      if (!f(x, i)) return;
      const uint32_t at = atomicAdd(&sh.n_list, 1u);
      if (at < (uint32_t)kSampleList) sh.list[at] = entry(x, i);
    });
    __syncthreads();
    return sh.n_list;
  }

  // ---- the cut behind which less than `need` (of tokens, or of weight) stands
  // before a token, among those that `within` keeps.  The values' range is cut into
  // bins, the bin that holds the cut becomes the range, until its tokens fit the
  // list or are all equal.
  // (in 64 bits: no difference of two logits overflows or vanishes)
  __device__ __forceinline__ static int bin_of(float x, float hi, double scale) {
    return min(kSampleBins - 1, (int)(((double)hi - (double)x) * scale));
  }
  __device__ Cut cut(bool by_weight, u64 need, float lo, float hi, const Cut& within) {
    u64 above = 0;
    for (;;) {
      const double scale = hi > lo ? (double)(kSampleBins - 1) / ((double)hi - (double)lo) : 0.;
      for (int i = tid; i < kSampleBins; i += NT) { sh.mass[i] = 0; sh.count[i] = 0; }
      __syncthreads();
      each([&](float x, int i) {
        if (!(x >= lo && x <= hi && within.keeps(x, i))) return;
        const int b = bin_of(x, hi, scale);
        atomicAdd(&sh.count[b], 1u);
        if (by_weight) atomicAdd(&sh.mass[b], weigh(x));
      });
      __syncthreads();
      constexpr int PER = kSampleBins / NT;
      u64 mine = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) mine += by_weight ? sh.mass[tid * PER + i] : sh.count[tid * PER + i];
      u64 total;
      u64 at = above + before(mine, &total);
      if (at < need && at + mine >= need) {
        for (int i = 0; i < PER; ++i) {
          const u64 c = by_weight ? sh.mass[tid * PER + i] : sh.count[tid * PER + i];
          if (at + c >= need) {
            sh.word[0] = tid * PER + i;
            sh.word[1] = at;
            break;
          }
          at += c;
        }
      } else if (tid == 0 && above + total < need) {      // all of them stay
        sh.word[0] = kSampleBins;
      }
      __syncthreads();
      const int bin = (int)sh.word[0];
      if (bin >= kSampleBins) return within;
      above = sh.word[1];
      auto inside = [&](float x, int i) {
        return x >= lo && x <= hi && within.keeps(x, i) && bin_of(x, hi, scale) == bin;
      };
      const uint32_t n = sh.count[bin];
      __syncthreads();
      if (n <= (uint32_t)kSampleList) {
        collect(inside);
        sort(sh.list, (int)n);
        u64 w[kSampleList / NT], sum = 0;
#pragma unroll
        for (int i = 0; i < kSampleList / NT; ++i) {
          const int p = tid * (kSampleList / NT) + i;
          w[i] = p >= (int)n ? 0 : by_weight ? weigh(entry_value(sh.list[p])) : 1;
          sum += w[i];
        }
        u64 b = above + before(sum, &total);
#pragma unroll
        for (int i = 0; i < kSampleList / NT; ++i) {
          const int p = tid * (kSampleList / NT) + i;
          // the last one with less than `need` before it
          if (p < (int)n && b < need && (b + w[i] >= need || p == (int)n - 1)) sh.word[2] = sh.list[p];
          b += w[i];
        }
        __syncthreads();
        const u64 e = sh.word[2];
        __syncthreads();
        return Cut{entry_value(e), entry_index(e)};
      }
      float least = INFINITY, most = -INFINITY;
      each([&](float x, int i) {
        if (inside(x, i)) { least = fminf(least, x); most = fmaxf(most, x); }
      });
      reduce_range(least, most);
      if (least == most) {
        // equal ones: the first of them, by index
        const u64 w = by_weight ? weigh(most) : 1;
        const u64 take = (need - above + w - 1) / w;
        return Cut{most, index_of_equal(most, take, within)};
      }
      lo = least;
      hi = most;
    }
  }
  __device__ __forceinline__ void reduce_range(float& least, float& most) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      least = fminf(least, __shfl_xor(least, o));
      most = fmaxf(most, __shfl_xor(most, o));
    }
    __syncthreads();
    if (lane == 0) { sh.range[wave] = least; sh.range[kSampleWaves + wave] = most; }
    __syncthreads();
    for (int i = 0; i < kSampleWaves; ++i) {
      least = fminf(least, sh.range[i]);
      most = fmaxf(most, sh.range[kSampleWaves + i]);
    }
  }

  // ---- pieces of the row in order: wave w's part of piece j is entry j * waves +
  // w of sums.  The index of the token in which the running sum of f passes `target`
  // (the first with more than `target` up to it), of f's values given the sums.
  template <typename F>
  __device__ __forceinline__ u64 sum_pieces(F&& f) {
    const int n = pieces();
    __syncthreads();
    u64 mine = 0;
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      float x[VEC];
      load(j, tid, x);
      u64 t = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (x[e] > -INFINITY) t += f(x[e], (j * NT + tid) * VEC + e);
      mine += t;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
      if (lane == 0) sh.sums[j * kSampleWaves + wave] = t;
    }
    return all(mine);
  }
  template <typename F>
  __device__ __forceinline__ int locate(u64 target, F&& f) {
    const int n = pieces() * kSampleWaves, per = (n + NT - 1) / NT;
    u64 mine = 0, total;
    for (int i = tid * per; i < min(n, tid * per + per); ++i) mine += sh.sums[i];
    u64 at = before(mine, &total);
    if (at <= target && at + mine > target) {
      int i = tid * per;
      while (at + sh.sums[i] <= target) at += sh.sums[i++];
      sh.word[0] = i;
      sh.word[1] = at;
    }
    __syncthreads();
    const int p = (int)sh.word[0];
    at = sh.word[1];
    if (wave == 0) {
      const int j = p / kSampleWaves, thread = p % kSampleWaves * 64 + lane;
      float x[VEC];
      load(j, thread, x);
      u64 w[VEC], t = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        w[e] = x[e] > -INFINITY ? f(x[e], (j * NT + thread) * VEC + e) : 0;
        t += w[e];
      }
      u64 incl = t;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const u64 y = __shfl_up(incl, o);
        if (lane >= o) incl += y;
      }
      u64 b = at + incl - t;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (b <= target && b + w[e] > target) sh.word[2] = (j * NT + thread) * VEC + e;
        b += w[e];
      }
    }
    __syncthreads();
    const int r = (int)sh.word[2];
    __syncthreads();
    return r;
  }
  __device__ __forceinline__ int index_of_equal(float v, u64 take, const Cut& within) {
    auto one = [&](float x, int i) -> u64 { return x == v && within.keeps(x, i); };
    sum_pieces(one);
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

  // ---- everything on a list of the first n tokens (all that may stay).  total: the
  // weight that top-p is a share of (0: that of the first k of the list).
  __device__ void from_list(int n, u64 k, float top_p, double min_weight, u64 total, float u,
                            int* token, u64* token_weight, u64* kept_weight) {
    constexpr int PER = kSampleList / NT;
    sort(sh.list, n);
    if (k > 0 && k < (u64)n) n = (int)k;
    u64 w[PER], sum = 0, all_of_list;
    bool large[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = tid * PER + i;
      const double v = p < n ? weigh.scaled(entry_value(sh.list[p])) : 0.;
      w[i] = Weigher::whole(v);
      large[i] = p < n && (p == 0 || v >= min_weight);
      sum += w[i];
    }
    u64 b = before(sum, &all_of_list);
    const u64 share = top_p < 1.f ? share_of(top_p, total ? total : all_of_list) : ~0ull;
    uint32_t stay = 0;
    u64 weight = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = tid * PER + i;
      if (large[i] && (p == 0 || b < share)) {
        ++stay;
        weight += w[i];
      }
      b += w[i];
    }
    const int kept = (int)all(stay);
    const u64 kept_sum = all(weight);
    // by index: the entries of those that stay, turned around
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = tid * PER + i;
      if (p < kept) sh.weight[p] = (u64)(uint32_t)sh.list[p] << 32 | (uint32_t)p;
    }
    __syncthreads();
    sort(sh.weight, kept);                 // (descending in ~index: ascending in index)
    u64 q[PER];
    sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = tid * PER + i;
      q[i] = p < kept ? weigh(entry_value(sh.list[(uint32_t)sh.weight[p]])) : 0;
      sum += q[i];
    }
    u64 t;
    u64 at = before(sum, &t);
    const u64 target = target_of(u, kept_sum);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int p = tid * PER + i;
      if (at <= target && at + q[i] > target) sh.word[3] = sh.list[(uint32_t)sh.weight[p]];
      at += q[i];
    }
    __syncthreads();
    const u64 e = sh.word[3];
    *token = entry_index(e);
    *token_weight = order_of(entry_value(e));
    *kept_weight = kept_sum;
  }
};

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  using S = Sampler<T>;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
  const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
  const float min_p = a.min_ps ? a.min_ps[r] : a.min_p;
  const int k_in = a.top_ks ? a.top_ks[r] : a.top_k;
  const float u = a.u[r];
  S s{sh, static_cast<const T*>(a.logits) + (int64_t)r * a.stride, a.vocab, false, false, Weigher{},
      tid, lane, wave};
  s.vectors = reinterpret_cast<uintptr_t>(s.row) % (4 * sizeof(T)) == 0;
  const int shift = a.vocab <= (1 << 18) ? 44 : 42;
  if (tid < 256) sh.table[tid] = ldexp(exp2((double)tid / 256.), shift);

  // ---- the largest and the smallest logit; this thread's largest
  float most = -INFINITY, least = INFINITY;
  int at = 0x7fffffff;
  s.each([&](float x, int i) {
    if (x > most) { most = x; at = i; }
    least = fminf(least, x);
  });
  const float mine = most;
  u64 best = most > -INFINITY ? S::entry(most, at) : 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const u64 y = __shfl_xor(best, o);
    best = y > best ? y : best;
  }
  if (lane == 0) sh.list[wave] = best;
  s.reduce_range(least, most);
  for (int i = 0; i < kSampleWaves; ++i) best = sh.list[i] > best ? sh.list[i] : best;
  __syncthreads();
  auto answer = [&](int token, float log_p) {
    if (tid != 0) return;
    a.tokens[r] = token;
    if (a.log_probs) a.log_probs[r] = log_p;
  };
  if (best == 0) return answer(-1, -INFINITY);
  // (a NaN among the settings leaves the first token)
  if (!(temperature > 0.f) || k_in == 1 || !(top_p > 0.f) || !(min_p <= 1.f))
    return answer(S::entry_index(best), 0.f);
  s.infinite = most == INFINITY;
  const float top = s.infinite ? 0.f : most;
  if (s.infinite) least = 0.f;
  s.weigh = Weigher{sh.table, (double)top, 256. * 1.4426950408889634074 / (double)temperature};
  const u64 k = k_in <= 0 || k_in >= a.vocab ? 0 : (u64)k_in;
  const double one = ldexp(1., shift), min_weight = min_p > 0.f ? (double)min_p * one : 0.;
  auto finish = [&](int token, float x, u64 total) {
    answer(token, (float)(((double)x - (double)top) / (double)temperature - log((double)total / one)));
  };

  // ---- few tokens can stay: a list
  int n_list = -1;
  if (a.vocab <= kSampleList) {
    n_list = (int)s.collect([](float, int) { return true; });
  } else if (k > 0 && k <= 512 && !s.infinite) {
    // the k-th largest of the threads' largest: at least k tokens are not below it.
    // lo: a bound that k threads reach
    uint32_t lo = 0, hi = order_of(most);
    const uint32_t key = order_of(mine);
    for (int i = 0; i < 20 && lo < hi; ++i) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      const u64 c = s.all(key >= mid && mine > -INFINITY);
      if (c >= k) {
        lo = mid;
        if (c == k) break;
      } else {
        hi = mid - 1;
      }
    }
    const uint32_t n = s.collect([&](float x, int) { return order_of(x) >= lo; });
    if (n <= (uint32_t)kSampleList) n_list = (int)n;
  }
  int token;
  u64 value, total;
  if (n_list >= 0) {
    s.from_list(n_list, k, top_p, min_weight, 0, u, &token, &value, &total);
    return finish(token, value_of((uint32_t)value), total);
  }
  // ---- many: where they end, then their sums in order of the index
  Cut cut;
  if (k > 0) cut = s.cut(false, k, least, top, cut);
  if (top_p < 1.f) {
    u64 sum = 0;
    s.each([&](float x, int i) { if (cut.keeps(x, i)) sum += s.weigh(x); });
    const u64 of = s.all(sum);
    // (no token below lo can stay: all of them together weigh less than 1 - top_p)
    const float lo = top + temperature * (logf((1.f - top_p) / (float)a.vocab) - 0.01f);
    cut = s.cut(true, S::share_of(top_p, of), fmaxf(least, lo), top, cut);
  }
  auto weight = [&](float x, int i) -> u64 {
    if (!cut.keeps(x, i)) return 0;
    const double v = s.weigh.scaled(x);
    return v >= min_weight ? Weigher::whole(v) : 0;
  };
  total = s.sum_pieces(weight);
  token = s.locate(S::target_of(u, total), weight);
  if (tid == 0) {
    float x = to_f32(s.row[token]);
    if (s.infinite) x = 0.f;
    finish(token, x, total);
  }
}

template <typename T>
hipError_t sample(const SampleArgs& a, hipStream_t s) {
  CR_LAUNCH((sample_kernel<T>), dim3(a.n_rows), dim3(kSampleThreads), 0, s, a);
  return hipGetLastError();
}
template hipError_t sample<bf16>(const SampleArgs&, hipStream_t);
template hipError_t sample<float>(const SampleArgs&, hipStream_t);

}  // namespace cr
