// Device code that the kernels over a paged cache share: lengths, LDS rows,
// capped scores (gfx950).
#pragma once
#include "serve.h"

namespace cr {

constexpr float kLog2e = 1.4426950408889634f;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A sequence's length: its queries' slots count from it, but keys lie only in
// slots below max_len.
__device__ __forceinline__ int seq_len(const PagedSeqs& p, int s) { return max(p.lens[s], 0); }

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

// This lane's number, from no register that has to live.  (opaque: not merged
// with an earlier one)
__device__ __forceinline__ int lane_again() {
  int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(l));
  return l;
}

}  // namespace cr
