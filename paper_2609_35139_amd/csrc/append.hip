// Appends the keys and values of new tokens to a paged cache, keys and queries
// rotated to their positions on the way (gfx950).
#include <algorithm>
#include <cmath>

#include "serve.h"

namespace cr {

// Sequences of one launch, by value: query offsets of sequences
// [first, first + count], or (offsets unused) q queries for every sequence.
constexpr int kAppendSeqs = 256;
struct AppendBatch {
  int first, count, q;
  int offs[kAppendSeqs + 1];
};

// A thread rotates 8 rotate-half pairs (i0 .. i0 + 7 and their partners) of
// HPT heads of one token: its eight angles serve all of them.  The angle
// p f_i is formed in turns in fp64 and reduced to half a turn, its cosine and
// sine are fp64 and rounded to 32 bits once, as in the repair's own rotation
// (fp32 functions of the reduced angle: 55.5 instead of 56.1 us at 11,000 tokens,
// 5.0 instead of 5.1 at 64, and an error of 3.0e-8 instead of 1.9e-8 of fp32
// keys).  Grid y = 1 copies the values, 8 elements of one head per thread.
// Bound by memory: each element is read and written once, 16 bytes at a time.
// 11,243 tokens of 32 + 8 heads of 128 (276 MB with the values) take 56 us, 4.9
// TB/s; 64 single tokens take 5.1 us, which is a launch and two dependent reads.
template <typename T, int HPT>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, KeyRope kr, AppendBatch b) {
  const int per_head = blockIdx.y == 0 ? a.head_dim / 16 : a.head_dim / 8;
  const int q_heads = a.q ? a.n_heads : 0;
  const int heads = blockIdx.y == 0 ? a.n_kv + q_heads : a.n_kv;
  const int groups = blockIdx.y == 0 ? (heads + HPT - 1) / HPT : heads;
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per_token = groups * per_head;
  const int64_t t64 = idx / per_token;
  const int t_first = b.q ? 0 : b.offs[0], t_end = b.q ? a.n_tokens : b.offs[b.count];
  if (t64 >= t_end - t_first) return;
  const int t = t_first + (int)t64;
  const int rem = (int)(idx - t64 * per_token);
  const int hg = rem / per_head, c0 = (rem - hg * per_head) * 8;
  int s, nq, i;
  if (b.q) {
    s = t / b.q;
    nq = b.q;
    i = t - s * b.q;
  } else {
    int lo = 0, hi = b.count;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (b.offs[mid] <= t) lo = mid; else hi = mid;
    }
    s = b.first + lo;
    nq = b.offs[lo + 1] - b.offs[lo];
    i = t - b.offs[lo];
  }
  const PagedSeqs& ps = a.seqs;
  const int slot = max(ps.lens[s], 0) - nq + i;
  int64_t row = -1;                      // element offset of the token's row, -1: dropped
  if (slot >= 0 && slot < ps.max_len) {
    const int id = ps.table[(int64_t)s * ps.max_blocks + (slot >> ps.shift)];
    if (id >= 0 && id < ps.n_blocks)
      row = (int64_t)id * ps.block + (int64_t)(slot & ((1 << ps.shift) - 1)) * ps.token;
  }
  if (blockIdx.y == 1) {
    if (row < 0) return;
    Vec8<T> x;
    x.load(static_cast<const T*>(a.v) + (int64_t)t * a.v_token + (int64_t)hg * a.v_head + c0);
    x.store(static_cast<T*>(a.v_cache) + row + (int64_t)hg * ps.head + c0);
    return;
  }
  const int half = a.head_dim / 2;
  float cs[8], sn[8];
  if (a.rotate) {
    const double p = a.positions ? (double)a.positions[t] : (double)slot;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = p * kr.f[c0 + e];
      double s, c;
      sincospi(2. * (turns - rint(turns)), &s, &c);
      cs[e] = (float)(kr.scale * c);
      sn[e] = (float)(kr.scale * s);
    }
  }
  // heads [0, n_kv) are keys, the others queries; a head is loaded before the
  // one ahead of it is stored (a dropped token's keys are loaded all the same)
  const int h0 = hg * HPT, h1 = min(h0 + HPT, heads);
  auto src = [&](int h) {
    return (h < a.n_kv ? static_cast<const T*>(a.k) + (int64_t)t * a.k_token + (int64_t)h * a.k_head
                       : static_cast<const T*>(a.q) + (int64_t)t * a.q_token +
                             (int64_t)(h - a.n_kv) * a.q_head) + c0;
  };
  Vec8<T> x, y;
  x.load(src(h0));
  y.load(src(h0) + half);
  for (int h = h0; h < h1; ++h) {
    Vec8<T> nx, ny;
    const T* next = src(min(h + 1, h1 - 1));
    nx.load(next);
    ny.load(next + half);
    if (a.rotate) {
      float f1[8], f2[8];
      x.to_float(f1);
      y.to_float(f2);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = f1[e], w = f2[e];
        f1[e] = cs[e] * u - sn[e] * w;
        f2[e] = cs[e] * w + sn[e] * u;
      }
      x.from_float(f1);
      y.from_float(f2);
    }
    T* dst = (h < a.n_kv ? static_cast<T*>(a.k_cache) + row + (int64_t)h * ps.head
                         : static_cast<T*>(a.q_out) + (int64_t)t * a.o_token +
                               (int64_t)(h - a.n_kv) * a.o_head) + c0;
    if (h >= a.n_kv || row >= 0) {
      x.store(dst);
      y.store(dst + half);
    }
    x = nx;
    y = ny;
  }
}

template <typename T>
hipError_t append_kv(const AppendArgs& a, const KeyRope& kr_in, const int32_t* off,
                     hipStream_t s) {
  if (a.n_tokens <= 0) return hipSuccess;
  KeyRope kr = kr_in;                       // radians per position -> turns
  for (int i = 0; i < kr.half; ++i) kr.f[i] = kr.f[i] / (2.0 * M_PI);
  const int heads = a.n_kv + (a.q ? a.n_heads : 0);
  auto launch = [&](const AppendBatch& b, int tokens) {
    const int64_t groups = append_groups(tokens, a.n_kv, heads, a.head_dim);
    if (!fits_launch(groups, 256)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)groups, 2);
    if (append_heads(tokens, heads, a.head_dim) == 1) {
      CR_LAUNCH((append_kernel<T, 1>), grid, dim3(256), 0, s, a, kr, b);
    } else {
      CR_LAUNCH((append_kernel<T, 4>), grid, dim3(256), 0, s, a, kr, b);
    }
    return hipGetLastError();
  };
  AppendBatch b{};
  if (!off) {
    b.q = a.n_tokens / a.seqs.n_seqs;
    return launch(b, a.n_tokens);
  }
  for (int s0 = 0; s0 < a.seqs.n_seqs; s0 += kAppendSeqs) {
    b.first = s0;
    b.count = std::min(kAppendSeqs, a.seqs.n_seqs - s0);
    for (int i = 0; i <= b.count; ++i) b.offs[i] = off[s0 + i];
    const int tokens = b.offs[b.count] - b.offs[0];
    if (tokens == 0) continue;
    const hipError_t e = launch(b, tokens);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template hipError_t append_kv<bf16>(const AppendArgs&, const KeyRope&, const int32_t*, hipStream_t);
template hipError_t append_kv<float>(const AppendArgs&, const KeyRope&, const int32_t*, hipStream_t);

}  // namespace cr
