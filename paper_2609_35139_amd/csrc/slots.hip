// The slots of a paged cache that stay when a sequence is over its budget, and
// their compaction (gfx950).
#include <algorithm>

#include "answer.h"

namespace cr {

// ------------------------------------------------------------------- choose
// A sequence of n slots keeps m = min(n, budget): its last min(recent, m), its
// first min(first, what is left), and of the others those of the largest weight,
// the lowest slot of equal ones.  Weights as whole numbers in their order: the
// sign bit turned over, or all bits of a negative one; NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (!(w > -INFINITY)) w = -INFINITY;            // NaN
  const uint32_t b = __float_as_uint(w + 0.f);    // -0 + 0 = 0
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// Sum over the lanes before this one and over all lanes of a wave.
__device__ __forceinline__ uint32_t lanes_before(uint32_t v, int lane, uint32_t* total) {
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  *total = __shfl(x, 63);
  return x - v;
}

constexpr int kChooseBins = 2048;

// A workgroup chooses for one (layer, sequence, head), each wave in a run of slots of
// its own.  The smallest weight that stays is found by counting: the weights' range is
// cut into at most 2048 bins and the bin that holds the last one to stay becomes the
// range, until its weights are few enough to compare each with each, or all equal.
// EPT: vectors of four slots that a thread keeps in registers; 0: as many as there are,
// read again from the caches in every pass.
template <int NT, int EPT>
__global__ __launch_bounds__(NT) void choose_kernel(ChooseArgs a) {
  constexpr int WAVES = NT / 64;
  constexpr uint32_t FEW = 256;
  // (every bin COPIES times, for a lane each: lanes that count in the same one wait for
  // each other)
  constexpr int COPIES = NT == 256 ? 2 : 4;
  typedef uint32_t Counts __attribute__((ext_vector_type(COPIES)));
  __shared__ Counts hist[kChooseBins];
  __shared__ __align__(16) uint32_t few[FEW];
  // (the list's counts have a place of their own: where all weights are equal, no barrier
  // lies between the last look at the range in `scratch` and the first count)
  __shared__ uint32_t scratch[WAVES * 2], counts[WAVES * 2], found[3];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int head = blockIdx.x % a.n_kv, ls = blockIdx.x / a.n_kv;
  const int s = ls % a.n_seqs, layer = ls / a.n_seqs;
  const int n = min(max(a.lens[s], 0), a.max_len);
  const int budget = a.budgets ? min(max(a.budgets[s], 0), a.budget) : a.budget;
  const int m = min(n, budget);
  int* out = a.kept + (int64_t)blockIdx.x * a.budget;
  if (layer == 0 && head == 0 && tid == 0) a.kept_lens[s] = m;
  for (int i = m + tid; i < a.budget; i += NT) out[i] = -1;
  const int recent = min(a.recent, m), first = min(a.first, m - recent), need = m - first - recent;
  if (n == m || need == 0) {
    for (int i = tid; i < m; i += NT) out[i] = i < first || n == m ? i : n - m + i;
    return;
  }
  const int lo = first, hi = n - recent;          // the slots to choose from: more than need
  const float* w = a.weights.data + (int64_t)layer * a.weights.layer + (int64_t)s * a.weights.seq +
                   (int64_t)head * a.weights.head;
  const bool vectors = reinterpret_cast<uintptr_t>(w) % 16 == 0;
  const int run = (n + 256 * WAVES - 1) / (256 * WAVES);   // vectors of a lane, 256 slots each
  auto slot_of = [&](int j) { return ((wave * run + j) * 64 + lane) * 4; };
  uint4 keep[EPT ? EPT : 1];
  // (a slot that is not to be chosen from has key 0, below that of every weight)
  auto load = [&](int j) {
    const int i = slot_of(j), i0 = i - lane * 4;
    uint4 k{0, 0, 0, 0};
    if (i0 >= lo && i0 + 256 <= hi && vectors) {
      const float4 x = *reinterpret_cast<const float4*>(w + i);
      k = uint4{weight_key(x.x), weight_key(x.y), weight_key(x.z), weight_key(x.w)};
    } else if (i0 < hi && i0 + 256 > lo) {
      k.x = i >= lo && i < hi ? weight_key(w[i]) : 0u;
      k.y = i + 1 >= lo && i + 1 < hi ? weight_key(w[i + 1]) : 0u;
      k.z = i + 2 >= lo && i + 2 < hi ? weight_key(w[i + 2]) : 0u;
      k.w = i + 3 >= lo && i + 3 < hi ? weight_key(w[i + 3]) : 0u;
    }
    return k;
  };
  if constexpr (EPT > 0) {
#pragma unroll
    for (int j = 0; j < EPT; ++j)
      if (j < run) keep[j] = load(j);
  }
  // f(vector of keys, its first slot), vector by vector of this thread
  auto each_vector = [&](auto&& f) {
    if constexpr (EPT > 0) {
#pragma unroll
      for (int j = 0; j < EPT; ++j)
        if (j < run) f(keep[j], slot_of(j));
    } else {
      constexpr int U = 4;                        // (the next ones on their way meanwhile)
      uint4 k[U], next[U];
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = load(min(u, run - 1));
#pragma unroll 1
      for (int j = 0; j < run; j += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) k[u] = next[u];
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = load(min(j + U + u, run - 1));
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (j + u < run) f(k[u], slot_of(j + u));
      }
    }
  };
  // f(key) for this thread's slots
  auto each = [&](auto&& f) {
    each_vector([&](const uint4& k, int) {
      f(k.x);
      f(k.y);
      f(k.z);
      f(k.w);
    });
  };
  // the range of the keys (0 is no key: it becomes the largest number)
  uint32_t kmin = ~0u, kmax = 0;
  each([&](uint32_t k) { kmin = min(kmin, k - 1u); kmax = max(kmax, k); });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    kmin = min(kmin, (uint32_t)__shfl_xor(kmin, o));
    kmax = max(kmax, (uint32_t)__shfl_xor(kmax, o));
  }
  if (lane == 0) { scratch[wave] = kmin; scratch[WAVES + wave] = kmax; }
  __syncthreads();
  for (int i = 0; i < WAVES; ++i) {
    kmin = min(kmin, scratch[i]);
    kmax = max(kmax, scratch[WAVES + i]);
  }
  kmin += 1u;
  auto count_of = [&](int bin) {
    const Counts c = hist[bin];
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < COPIES; ++i) t += c[i];
    return t;
  };
  // the key of the last one to stay (kmin in the end), and how many of that key stay
  uint32_t left = need;
  while (kmin < kmax) {
    const uint32_t span = kmax - kmin;
    const int bits = 32 - __clz(span), sh = bits > 11 ? bits - 11 : 0;
    for (int i = tid; i < kChooseBins; i += NT) hist[i] = Counts{};
    if (tid < (int)FEW) few[tid] = 0;               // (0 is no key)
    if (tid == 0) found[2] = 0;
    __syncthreads();
    each([&](uint32_t k) {
      if (k - kmin <= span)
        atomicAdd(reinterpret_cast<uint32_t*>(hist) + ((k - kmin) >> sh) * COPIES + lane % COPIES, 1u);
    });
    __syncthreads();
    // bins from the highest down: the first whose running count reaches `left`
    constexpr int PER = kChooseBins / NT;
    uint32_t c[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine += c[i] = count_of(kChooseBins - 1 - (tid * PER + i));
    uint32_t total;
    uint32_t before = lanes_before(mine, lane, &total);
    if (lane == 0) scratch[wave] = total;
    __syncthreads();
    for (int i = 0; i < wave; ++i) before += scratch[i];
    if (before < left && before + mine >= left) {   // one thread
      bool done = false;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (done) continue;
        done = before + c[i] >= left;
        if (done) {
          found[0] = kChooseBins - 1 - (tid * PER + i);
          found[1] = left - before;
        } else {
          before += c[i];
        }
      }
    }
    __syncthreads();
    const uint32_t to_bin = found[0] << sh, count = count_of(found[0]);
    left = found[1];
    kmax = kmin + to_bin + min(span - to_bin, (1u << sh) - 1u);
    kmin += to_bin;
    if (count <= FEW && kmin < kmax) {
      const uint32_t range = kmax - kmin;
      each_vector([&](const uint4& k, int) {
        const bool any = (k.x - kmin <= range) | (k.y - kmin <= range) | (k.z - kmin <= range) |
                         (k.w - kmin <= range);
        if (!__any(any)) return;
        const uint32_t v[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v[e] - kmin <= range) few[atomicAdd(&found[2], 1u)] = v[e];
      });
      __syncthreads();
      if (tid < (int)count) {
        const uint32_t k = few[tid];
        uint32_t above = 0, equal = 0;
#pragma unroll 4
        for (uint32_t i = 0; i < count; i += 4) {
          const uint4 o = *reinterpret_cast<const uint4*>(few + i);
          above += (o.x > k) + (o.y > k) + (o.z > k) + (o.w > k);
          equal += (o.x == k) + (o.y == k) + (o.z == k) + (o.w == k);
        }
        if (above < left && above + equal >= left) {   // (equal ones write the same)
          found[0] = k;
          found[1] = left - above;
        }
      }
      __syncthreads();
      kmin = kmax = found[0];
      left = found[1];
    }
    __syncthreads();
  }
  // ---- the list, in order of the slots: a slot's place is the number of those
  // before it that stay whatever happens, and of the equal ones up to `left`.  Counted
  // for each wave's run, then written run by run.
  // the lanes whose slot e of a vector stays whatever happens, or is an equal one
  struct Marks { uint64_t sure[4], equal[4]; };
  auto marks_of = [&](const uint4& k, int i) {
    const uint32_t v[4] = {k.x, k.y, k.z, k.w};
    Marks r;
    const bool inside = i - lane * 4 >= lo && i - lane * 4 + 256 <= hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.sure[e] = __ballot(v[e] > kmin);
      r.equal[e] = __ballot(v[e] == kmin);
      if (!inside) r.sure[e] |= __ballot(v[e] == 0 && i + e < n);
    }
    return r;
  };
  uint32_t sure_at = 0, equal_at = 0;
  each_vector([&](const uint4& k, int i) {
    const Marks r = marks_of(k, i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sure_at += __popcll(r.sure[e]);
      equal_at += __popcll(r.equal[e]);
    }
  });
  if (lane == 0) { counts[wave] = sure_at; counts[WAVES + wave] = equal_at; }
  __syncthreads();
  sure_at = equal_at = 0;
  for (int i = 0; i < wave; ++i) { sure_at += counts[i]; equal_at += counts[WAVES + i]; }
  each_vector([&](const uint4& k, int i) {
    const Marks r = marks_of(k, i);
    // those of the lanes before this one, of all four slots
    uint32_t at = sure_at, eq = equal_at;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      at = __builtin_amdgcn_mbcnt_hi((uint32_t)(r.sure[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)r.sure[e], at));
      eq = __builtin_amdgcn_mbcnt_hi((uint32_t)(r.equal[e] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)r.equal[e], eq));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is_sure = (r.sure[e] >> lane) & 1, is_equal = (r.equal[e] >> lane) & 1;
      if (is_sure | (is_equal & (eq < left))) out[at + min(eq, left)] = i + e;
      at += is_sure;
      eq += is_equal;
      sure_at += __popcll(r.sure[e]);
      equal_at += __popcll(r.equal[e]);
    }
  });
}

hipError_t choose(const ChooseArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.n_layers * a.n_seqs * a.n_kv));
  // 256 threads hold 8,192 slots in registers, 512 hold 32,768.  Where there are more than
  // two workgroups for a CU, small ones fill it better (2,304 rows of 8,000 slots of which
  // half stay: 44 us, with 512 threads 60; 520 rows 18.3 and 22.7), else large ones are done
  // sooner (512 rows: 15 us, with 256 threads 17; 288 rows 14 and 16).  Slots that are read
  // again in every pass take twice as long (2,304 rows of 30,000: 331 us, from registers
  // 152).  The rule goes by the table, as the lengths are on the device: rows of 4,000 slots
  // take 220 us in a table of 65,536 and 28 in one of 8,192.
  if (a.max_len <= 8192 && grid.x > 512) {
    CR_LAUNCH((choose_kernel<256, 8>), grid, dim3(256), 0, s, a);
  } else if (a.max_len <= 32768) {
    CR_LAUNCH((choose_kernel<512, 16>), grid, dim3(512), 0, s, a);
  } else {
    CR_LAUNCH((choose_kernel<1024, 0>), grid, dim3(1024), 0, s, a);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ compact
// A workgroup moves one component (keys, values) of one (layer, sequence, head): MOVE
// slots at a time, all read before any is written.  In place that is enough: the list
// ascends, so kept[i] >= i and what a step writes lies before all that later steps
// read.  So the next step's rows are on their way before this one's are written, and
// its addresses are looked up while this one's rows are on their way.
//
// A workgroup's part of a row has 2^LOG 16-byte chunks, a thread moves chunk tid % 2^LOG
// of U rows (rows that are no power of two: threads past the row idle).  Bound by
// memory where there are enough workgroups; few of them, in place, share the rows'
// columns, down to a cache line (36 layers of 2 heads, 2,048 of 4,096 slots of 256
// bytes: 55 us with whole rows, 41 with halves, several such caches in turn; 28 on one
// of them again and again, whose 153 MB stay in the last-level cache), out of place the
// steps.
template <int LOG>
struct MoveCfg {
  static constexpr int NT = 256, PER_ROW = 1 << LOG, RPP = NT / PER_ROW;   // rows per pass
  static constexpr int U = RPP > 32 ? NT / RPP : 8, MOVE = RPP * U;
  static_assert(MOVE <= NT, "a thread looks a row up");
};

// Slot j of a sequence: bytes from its pool, or -1.
__device__ __forceinline__ int64_t slot_bytes(const CompactArgs& a, const int* table, int j) {
  const int id = table[j >> a.seqs.shift];
  if (id < 0 || id >= a.seqs.n_blocks) return -1;
  return ((int64_t)id * a.seqs.block + (int64_t)(j & ((1 << a.seqs.shift) - 1)) * a.seqs.token) *
         a.element_bytes;
}

// The weights of one (layer, sequence, head), moved alike, and 0 behind them.
__device__ __forceinline__ void move_weights(const CompactArgs& a) {
  const int tid = threadIdx.x;
  const int head = blockIdx.x % a.n_kv, ls = blockIdx.x / a.n_kv;
  const int s = ls % a.seqs.n_seqs, layer = ls / a.seqs.n_seqs;
  const int n = min(max(a.seqs.lens[s], 0), a.seqs.max_len);
  const int m = min(max(a.kept_lens[s], 0), a.budget), end = min(m, a.seqs.max_len);
  const int* kept = a.kept + (int64_t)blockIdx.x * a.budget;
  float* w = a.weights.data + (int64_t)layer * a.weights.layer + (int64_t)s * a.weights.seq +
             (int64_t)head * a.weights.head;
  constexpr int U = 8;
  for (int i0 = 0; i0 < max(n, end); i0 += 256 * U) {
    float x[U];
    bool write[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 256 + tid;
      x[u] = 0.f;
      write[u] = i < n;                          // behind those that stay: nothing yet
      if (i < end) {
        const int j = kept[i];
        write[u] = j >= 0 && j < n;              // (no slot: it keeps what it holds)
        if (write[u]) x[u] = w[j];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+v"(x[u]));
    __syncthreads();                             // everything of this step is read
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (write[u]) w[i0 + u * 256 + tid] = x[u];
  }
}

template <int LOG>
__global__ __launch_bounds__(256) void compact_kernel(CompactArgs a) {
  using C = MoveCfg<LOG>;
  __shared__ int64_t src[2][C::MOVE], dst[2][C::MOVE];
  const int tid = threadIdx.x;
  const int head = blockIdx.x % a.n_kv, ls = blockIdx.x / a.n_kv;
  const int s = ls % a.seqs.n_seqs, layer = ls / a.seqs.n_seqs;
  const int comp = blockIdx.y;
  if (comp == 2) {
    if (blockIdx.z == 0) move_weights(a);
    return;
  }
  const int n = min(max(a.seqs.lens[s], 0), a.seqs.max_len);
  const int m = min(max(a.kept_lens[s], 0), a.budget);
  const int* kept = a.kept + (int64_t)blockIdx.x * a.budget;
  const int* table = a.seqs.table + (int64_t)s * a.seqs.max_blocks;
  const int* out = a.table_out ? a.table_out + (int64_t)s * a.max_blocks_out : table;
  const int most = min(m, a.max_blocks_out << a.seqs.shift);
  char* base = a.kv + ((int64_t)layer * a.layer + (int64_t)comp * a.kv_step +
                       (int64_t)head * a.seqs.head) * a.element_bytes;
  const int columns = a.table_out ? 1 : gridDim.z, shares = a.table_out ? gridDim.z : 1;
  const int chunk = (tid & (C::PER_ROW - 1)) + (columns > 1 ? blockIdx.z * C::PER_ROW : 0), r0 = tid >> LOG;
  const bool active = chunk * 16 < a.row_bytes;
  const int stride = C::MOVE * shares;           // (out of place the steps depend on nothing)
  auto look_up = [&](int i0, int st) {
    if (tid >= C::MOVE) return;
    int64_t from = -1, to = -1;
    const int i = i0 + tid;
    if (i < most) {
      const int j = kept[i];
      if (j >= 0 && j < n && (j != i || a.table_out)) {
        from = slot_bytes(a, table, j);
        to = slot_bytes(a, out, i);
      }
    }
    src[st][tid] = to < 0 ? -1 : from;
    dst[st][tid] = to;
  };
  uint4 x[C::U];
  auto read = [&](int st) {
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
      const int64_t from = src[st][r0 + u * C::RPP];
      if (active && from >= 0) x[u] = *reinterpret_cast<const uint4*>(base + from + chunk * 16);
    }
  };
  int i0 = shares > 1 ? blockIdx.z * C::MOVE : 0, st = 0;
  if (i0 >= most) return;
  look_up(i0, 0);
  __syncthreads();
  read(0);
  for (; i0 < most; i0 += stride, st ^= 1) {
    look_up(i0 + stride, st ^ 1);
    // (the rows have to be here, not on their way, when the others write)
#pragma unroll
    for (int u = 0; u < C::U; ++u) asm volatile("" : "+v"(x[u].x), "+v"(x[u].y), "+v"(x[u].z), "+v"(x[u].w));
    __syncthreads();                             // everything of this step is read
    uint4 y[C::U];
#pragma unroll
    for (int u = 0; u < C::U; ++u) y[u] = x[u];
    if (i0 + stride < most) read(st ^ 1);
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
      const int r = r0 + u * C::RPP;
      if (active && src[st][r] >= 0) *reinterpret_cast<uint4*>(base + dst[st][r] + chunk * 16) = y[u];
    }
    __syncthreads();                             // this step's addresses are idle
  }
}

template <int LOG>
hipError_t compact_as(const CompactArgs& a, int columns, hipStream_t s) {
  const int64_t rows = (int64_t)a.n_layers * a.seqs.n_seqs * a.n_kv;
  const int64_t steps = ((int64_t)a.budget + MoveCfg<LOG>::MOVE - 1) / MoveCfg<LOG>::MOVE;
  // out of place: about eight workgroups to a CU
  const int64_t z = a.table_out ? std::max<int64_t>(1, std::min(steps, 2048 / (2 * rows))) : columns;
  const dim3 grid((unsigned)rows, a.weights.data ? 3 : 2, (unsigned)z);
  CR_LAUNCH((compact_kernel<LOG>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t compact(const CompactArgs& a, hipStream_t s) {
  const int chunks = a.row_bytes / 16;           // 4 (bf16 heads of 32) to 64 (fp32 of 256)
  int log = 2, columns = 1;
  while ((1 << log) < chunks) ++log;
  const int64_t groups = 2 * (int64_t)a.n_layers * a.seqs.n_seqs * a.n_kv;
  while (!a.table_out && log > 3 && groups * columns < 512) {
    --log;
    columns *= 2;
  }
  switch (log) {
    case 2: return compact_as<2>(a, columns, s);
    case 3: return compact_as<3>(a, columns, s);
    case 4: return compact_as<4>(a, columns, s);
    case 5: return compact_as<5>(a, columns, s);
    default: return compact_as<6>(a, columns, s);
  }
}

}  // namespace cr
