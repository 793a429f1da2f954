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

// SPLIT: the four waves of a workgroup share a tile's rows; else each has tiles
// of its own.
template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(256) void weigh_kernel(WeighArgs a, WeighTable tab) {
  using MM = Mma16<T>;
  using frag = typename MM::frag;
  constexpr int KPL = MM::KPL, KSTEP = MM::KSTEP, QF = D / KSTEP;
  constexpr int KT = weigh_keys(sizeof(T), D), KA = KT / 16;
  __shared__ float part[SPLIT ? 4 * KT : 1];
  const int lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % a.n_kv;
  const int worker = SPLIT ? blockIdx.x / a.n_kv : blockIdx.x / a.n_kv * 4 + wave;
  const int workers = gridDim.x / a.n_kv * (SPLIT ? 1 : 4);
  const int S = a.seqs.n_seqs;

  // ---- this worker's tiles [t0, t1) of all sequences' tiles, in order
  const int first64 = lane < S ? key_tiles<KT>(a, tab, lane) : 0;
  auto tiles_at = [&](int s0) {
    return s0 == 0 ? first64 : s0 + lane < S ? key_tiles<KT>(a, tab, s0 + lane) : 0;
  };
  auto wave_total = [&](int x) {
    long long t = x;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
    return t;
  };
  long long total = 0;
  for (int s0 = 0; s0 < S; s0 += 64) total += wave_total(tiles_at(s0));
  const long long per = (total + workers - 1) / workers;
  long long t0 = worker * per;
  const long long t1 = min(total, t0 + per);
  if (t0 >= t1) return;                          // (uniform in a workgroup where it has a barrier)
  int s = 0;
  long long base = 0;                            // tiles before sequence s
  for (int s0 = 0; s0 < S; s0 += 64) {
    const int mine = tiles_at(s0);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long x = __shfl_up(incl, o);
      if (lane >= o) incl += x;
    }
    const unsigned long long hit = __ballot(mine > 0 && base + incl > t0);
    if (hit) {
      const int l = __ffsll(hit) - 1;
      s = s0 + l;
      base += __shfl(incl, l) - __shfl(mine, l);
      break;
    }
    base += __shfl(incl, 63);
  }
  s = __builtin_amdgcn_readfirstlane(s);

  const bool general = a.cap_log2 > 0.f || a.bias;
  const int shift = a.seqs.shift, page_mask = (1 << shift) - 1;
  const T* kbase = static_cast<const T*>(a.k) + (int64_t)head * a.seqs.head;
  int tile = __builtin_amdgcn_readfirstlane((int)(t0 - base));

  for (; t0 < t1; ++t0) {
    int n = min(seq_len(a.seqs, s), a.seqs.max_len);
    while (tile * KT >= n || queries_of(a, tab, s).nq == 0) {     // the next sequence with a tile
      if (++s >= S) return;
      tile = 0;
      n = min(seq_len(a.seqs, s), a.seqs.max_len);
    }
    const Queries qs = queries_of(a, tab, s);
    const int len = seq_len(a.seqs, s);
    const int k0 = tile * KT;
    // ---- the tile's keys
    frag kf[KA][QF];
    unsigned none[KA];                           // bit i: key i of the atom lies in no block
    const int* table = a.seqs.table + (int64_t)s * a.seqs.max_blocks;
#pragma unroll
    for (int x = 0; x < KA; ++x) {
      const int key = min(k0 + x * 16 + c16, n - 1);
      const int id = table[key >> shift];
      const bool ok = id >= 0 && id < a.seqs.n_blocks;
      none[x] = (unsigned)__ballot(!ok) & 0xffffu;
      const T* p = kbase + (ok ? (int64_t)id * a.seqs.block : 0) +
                   (int64_t)(key & page_mask) * a.seqs.token;
#pragma unroll
      for (int kk = 0; kk < QF; ++kk) kf[x][kk] = load_frag<T, frag>(p + kk * KSTEP + g * KPL);
    }
    unsigned bad = 0;
#pragma unroll
    for (int x = 0; x < KA; ++x) bad |= none[x];

    float sum[KA * 4];
#pragma unroll
    for (int x = 0; x < KA * 4; ++x) sum[x] = 0.f;

    // ---- the rows that see some of them
    const int n_rows = qs.nq * a.group;
    int r0 = 0;
    if (!a.hi) r0 = max(0, k0 - (len - qs.nq)) * a.group / 16 * 16;   // causal: from query k0 on
    if (SPLIT) r0 += wave * 16;
    for (; r0 < n_rows; r0 += SPLIT ? 64 : 16) {
      const int r = min(r0 + c16, n_rows - 1);
      const int i = r / a.group, hd = head * a.group + r - i * a.group;
      const int64_t t = qs.tok0 + i;
      int hi = max(min(a.hi ? a.hi[t] : len - qs.nq + i + 1, n), 0);
      int lo = a.lo ? max(a.lo[t], 0) : 0;
      const float lse = a.lse[t * a.n_kv * a.group + hd];
      // (a row that saw nothing weighs nothing)
      if (r0 + c16 >= n_rows || lse == -INFINITY) hi = lo = 0;
      if (!__any(lo < hi && lo < k0 + KT && hi > k0)) continue;
      const T* qp = static_cast<const T*>(a.q) + t * a.q_token + (int64_t)hd * a.q_head;
      frag qf[QF];
#pragma unroll
      for (int kk = 0; kk < QF; ++kk) qf[kk] = load_frag<T, frag>(qp + kk * KSTEP + g * KPL);
      // lse in exp2 units as the sum of two numbers, the second as a factor: one
      // rounding of a lse of 20 would put the whole row off by 2^-20
      const float ref = lse * kLog2e;
      const float rest = __builtin_fmaf(lse, kLog2e, -ref);
      const float factor = isfinite(rest) ? __builtin_amdgcn_exp2f(-rest) : 1.f;
      const bool whole = !bad && __all(lo <= k0 && hi >= k0 + KT);
      // exponents of an atom's scores where they are not just scaled
      auto capped = [&](f32x4& sc, int x) {
        const float slope = a.bias ? a.slopes_log2[hd] : 0.f;
        const int p = len - qs.nq + i;
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
          float y = sc[0] * a.scale_log2;
          if (a.cap_log2 > 0.f) {
            const float u = sc[0] * a.scale_over_cap;
            y = fabsf(u) > kCapSmall ? a.cap_log2 * tanh_of<T>(u) : y * tanh_over(u);
          }
          y -= slope * fabsf((float)(p - (k0 + x * 16 + 4 * g + e)));
          sc = f32x4{sc[1], sc[2], sc[3], y - ref};        // (turned once around)
        }
      };
#pragma unroll
      for (int x = 0; x < KA; ++x) {
        f32x4 sc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < QF; ++kk) sc = MM::mma(kf[x][kk], qf[kk], sc);
        if (general) {
          capped(sc, x);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[e] = __builtin_fmaf(sc[e], a.scale_log2, -ref);
        }
        f32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(sc[e]);
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = k0 + x * 16 + 4 * g + e;
            if (key < lo || key >= hi || ((none[x] >> (4 * g + e)) & 1)) w[e] = 0.f;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[x * 4 + e] = __builtin_fmaf(w[e], factor, sum[x * 4 + e]);
      }
    }
    // ---- one key per lane: atom x = id / 4, key 16 x + 4 g + id % 4, id = c16 % (4 KA)
    const float mine = sum_to_lane(sum, c16);
    const int id = c16 % (KA * 4), at = (id >> 2) * 16 + 4 * g + (id & 3);
    float* row = a.weights.data + (int64_t)s * a.weights.seq + (int64_t)head * a.weights.head;
    if (SPLIT) {
      if (c16 < KA * 4) part[wave * KT + at] = mine;
      __syncthreads();
      const int j = threadIdx.x;
      if (j < KT && k0 + j < n)
        row[k0 + j] += (part[j] + part[KT + j]) + (part[2 * KT + j] + part[3 * KT + j]);
      __syncthreads();
    } else if (c16 < KA * 4 && k0 + at < n) {
      row[k0 + at] += mine;
    }
    ++tile;
  }
}

template <typename T, int D>
hipError_t weigh_as(const WeighArgs& a, const WeighTable& tab, hipStream_t s) {
  // as many workers per KV head as there can be tiles, four waves to a SIMD at most
  constexpr int KT = weigh_keys(sizeof(T), D);
  const int64_t tiles = (int64_t)a.seqs.n_seqs * ((a.seqs.max_len + KT - 1) / KT);
  const int64_t most = (1024 + a.n_kv - 1) / a.n_kv;
  const int64_t groups = a.split ? tiles : (tiles + 3) / 4;
  const dim3 grid((unsigned)(a.n_kv * (groups < most ? groups : most)));
  if (a.split) {
    CR_LAUNCH((weigh_kernel<T, D, true>), grid, dim3(256), 0, s, a, tab);
  } else {
    CR_LAUNCH((weigh_kernel<T, D, false>), grid, dim3(256), 0, s, a, tab);
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
