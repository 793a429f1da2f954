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

// A workgroup chooses for one (layer, sequence, head).  The smallest weight that
// stays is found by counting: the weights' range is cut into at most 2048 bins,
// the bin that holds the last one to stay becomes the range, at most three times
// for 32 bits.  EPT: 4-slot groups that a thread keeps in registers; 0: as many
// as there are, read again from the caches in every pass.
template <int NT, int EPT>
__global__ __launch_bounds__(NT) void choose_kernel(ChooseArgs a) {
  constexpr int WAVES = NT / 64;
  __shared__ uint32_t hist[kChooseBins];
  __shared__ uint32_t scratch[WAVES * 2 + 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  const int groups = (hi + 4 * NT - 1) / (4 * NT);   // 4 NT slots each, from slot 0
  uint4 keep[EPT ? EPT : 1];
  auto load = [&](int j) {
    const int i = (j * NT + tid) * 4;
    uint4 k{0, 0, 0, 0};
    if (i < hi && i + 4 > lo) {
      float4 x;
      if (vectors && i + 4 <= a.max_len) {       // (may pass hi, not the row's end)
        x = *reinterpret_cast<const float4*>(w + i);
      } else {
        x.x = w[i];
        x.y = i + 1 < a.max_len ? w[i + 1] : 0.f;
        x.z = i + 2 < a.max_len ? w[i + 2] : 0.f;
        x.w = i + 3 < a.max_len ? w[i + 3] : 0.f;
      }
      k = uint4{weight_key(x.x), weight_key(x.y), weight_key(x.z), weight_key(x.w)};
    }
    return k;
  };
  if constexpr (EPT > 0) {
#pragma unroll
    for (int j = 0; j < EPT; ++j)
      if (j < groups) keep[j] = load(j);
  }
  // f(key, slot) for this thread's slots to choose from
  auto each = [&](auto&& f) {
    auto four = [&](const uint4& k, int j) {
      const int i = (j * NT + tid) * 4;
      const uint32_t v[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e >= lo && i + e < hi) f(v[e], i + e);
    };
    if constexpr (EPT > 0) {
#pragma unroll
      for (int j = 0; j < EPT; ++j)
        if (j < groups) four(keep[j], j);
    } else {
      for (int j = 0; j < groups; ++j) four(load(j), j);
    }
  };
  // the range of the keys
  uint32_t kmin = ~0u, kmax = 0;
  each([&](uint32_t k, int) { kmin = min(kmin, k); kmax = max(kmax, k); });
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
  // the key of the last one to stay, and how many of that key stay
  uint32_t left = need;
  while (kmin < kmax) {
    const uint32_t span = kmax - kmin;
    const int bits = 32 - __clz(span), sh = bits > 11 ? bits - 11 : 0;
    for (int i = tid; i < kChooseBins; i += NT) hist[i] = 0;
    __syncthreads();
    each([&](uint32_t k, int) {
      if (k >= kmin && k <= kmax) atomicAdd(&hist[(k - kmin) >> sh], 1u);
    });
    __syncthreads();
    // bins from the highest down: the first whose running count reaches `left`
    constexpr int PER = kChooseBins / NT > 0 ? kChooseBins / NT : 1;
    uint32_t c[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = kChooseBins - 1 - (tid * PER + i);
      c[i] = b >= 0 ? hist[b] : 0;
      mine += c[i];
    }
    uint32_t total;
    uint32_t before = lanes_before(mine, lane, &total);
    if (lane == 0) scratch[wave] = total;
    __syncthreads();
    for (int i = 0; i < wave; ++i) before += scratch[i];
    if (before < left && before + mine >= left) {   // one thread
      int i = 0;
      while (before + c[i] < left) before += c[i++];
      scratch[WAVES] = kChooseBins - 1 - (tid * PER + i);
      scratch[WAVES + 1] = left - before;
    }
    __syncthreads();
    const uint32_t bin = scratch[WAVES];
    left = scratch[WAVES + 1];
    const uint32_t to_bin = bin << sh;
    kmax = kmin + to_bin + min(span - to_bin, (1u << sh) - 1u);
    kmin += to_bin;
    __syncthreads();
  }
  // ---- the list, in order of the slots: a slot's place is the number of those
  // before it that stay whatever happens, and of the equal ones up to `left`
  uint32_t all_before = 0, equal_before = 0;
  const int last = (n + 4 * NT - 1) / (4 * NT);
  auto place = [&](const uint4& k, int j) {
    const int i = (j * NT + tid) * 4;
    const uint32_t v[4] = {k.x, k.y, k.z, k.w};
    uint32_t sure = 0, equal = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = i + e;
      const bool in = at >= lo && at < hi;
      if (at < n && (!in || v[e] > kmin)) sure |= 1u << e;
      if (in && v[e] == kmin) equal |= 1u << e;
    }
    uint32_t total;
    const uint32_t packed = lanes_before(__popc(sure) | __popc(equal) << 16, lane, &total);
    if (lane == 0) scratch[wave] = total;
    __syncthreads();
    uint32_t sure_at = all_before + (packed & 0xffff), equal_at = equal_before + (packed >> 16);
    for (int x = 0; x < WAVES; ++x) {
      const uint32_t t = scratch[x];
      if (x < wave) { sure_at += t & 0xffff; equal_at += t >> 16; }
      all_before += t & 0xffff;
      equal_before += t >> 16;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is_equal = (equal >> e) & 1;
      if ((sure >> e) & 1 || (is_equal && equal_at < left)) out[sure_at + min(equal_at, left)] = i + e;
      sure_at += (sure >> e) & 1;
      equal_at += is_equal;
    }
  };
  if constexpr (EPT > 0) {
#pragma unroll
    for (int j = 0; j < EPT; ++j)
      if (j < last) place(j < groups ? keep[j] : uint4{0, 0, 0, 0}, j);
  } else {
    for (int j = 0; j < last; ++j) place(j < groups ? load(j) : uint4{0, 0, 0, 0}, j);
  }
}

hipError_t choose(const ChooseArgs& a, hipStream_t s) {
  const int64_t rows = (int64_t)a.n_layers * a.n_seqs * a.n_kv;
  const dim3 grid((unsigned)rows);
  if (a.max_len <= 4096) {
    CR_LAUNCH((choose_kernel<256, 4>), grid, dim3(256), 0, s, a);
  } else if (a.max_len <= 16384) {
    CR_LAUNCH((choose_kernel<1024, 4>), grid, dim3(1024), 0, s, a);
  } else if (a.max_len <= 65536) {
    CR_LAUNCH((choose_kernel<1024, 16>), grid, dim3(1024), 0, s, a);
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
// bytes: 52 us with whole rows, XX with halves), out of place the steps.
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
  const int64_t steps = (a.budget + MoveCfg<LOG>::MOVE - 1) / MoveCfg<LOG>::MOVE;
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
