// Host-side argument checks and buffer layout helpers shared by the entry
// points (internal to the library).
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <vector>

#include "../../include/cacherepair.h"
#include "launch.h"

namespace cr {

constexpr uint64_t ALIGN = 256;
inline uint64_t align_up(uint64_t x, uint64_t a = ALIGN) { return (x + a - 1) / a * a; }
inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

struct Arena {
  uint64_t off = 0;
  uint64_t take(uint64_t bytes) {
    const uint64_t o = off;
    off = align_up(off + bytes);
    return o;
  }
};

inline size_t esize(int dtype) { return dtype == CR_DTYPE_F32 ? 4 : 2; }

inline cr_status check_dtype(const cr_kv_layout* l) {
  return (l->dtype == CR_DTYPE_BF16 || l->dtype == CR_DTYPE_F32) ? CR_OK : CR_ERR_DTYPE;
}

// Injective index map over (stride, extent) pairs: with the dims sorted by
// stride, each stride must exceed the largest offset reachable through the
// dims inside it.  The largest offset must also stay below 2^62 elements, so
// that no element offset a kernel forms in int64 can overflow.
struct Dim { int64_t s, e; };
// At most six (stride, extent) pairs: dim, head, token, (block,) K/V, layer.
// Fixed capacity, so validating a call allocates nothing.
struct Dims {
  Dim d[6];
  int n = 0;
  void push_back(Dim x) { d[n++] = x; }
};
inline cr_status check_injective(Dims dims) {
  std::sort(dims.d, dims.d + dims.n, [](const Dim& a, const Dim& b) { return a.s < b.s; });
  int64_t reach = 0;  // largest offset reachable by the dims visited so far
  for (int i = 0; i < dims.n; ++i) {
    const Dim& x = dims.d[i];
    if (x.s <= reach) return CR_ERR_LAYOUT;
    int64_t span;
    if (__builtin_mul_overflow(x.s, x.e - 1, &span) || __builtin_add_overflow(reach, span, &reach) ||
        reach >= ((int64_t)1 << 62))
      return CR_ERR_LAYOUT;
  }
  return CR_OK;
}

inline cr_status check_layout(const cr_kv_layout* l, int64_t n_tokens) {
  const int64_t st[4] = {l->stride_layer, l->stride_kv, l->stride_token, l->stride_head};
  const int64_t ext[4] = {l->n_layers, 2, n_tokens, l->n_kv_heads};
  Dims dims;
  dims.push_back({1, l->head_dim});
  for (int i = 0; i < 4; ++i) {
    if (st[i] < 0 || st[i] % 8 != 0) return CR_ERR_LAYOUT;
    if (ext[i] > 1) dims.push_back({st[i], ext[i]});
  }
  if (n_tokens == 0) return CR_OK;  // no element is addressed
  return check_injective(dims);
}

// Injectivity of a paged layout over (layer, kv, block, row, head, dim).
inline cr_status check_page_strides(const cr_kv_layout* l, int32_t bs, int32_t n_blocks,
                             int64_t stride_block) {
  if (bs < 1 || bs > 1024 || (bs & (bs - 1)) || n_blocks < 1) return CR_ERR_LAYOUT;
  if (stride_block < 0 || stride_block % 8) return CR_ERR_LAYOUT;
  const int64_t st[5] = {l->stride_layer, l->stride_kv, stride_block, l->stride_token,
                         l->stride_head};
  const int64_t ext[5] = {l->n_layers, 2, n_blocks, bs, l->n_kv_heads};
  Dims dims;
  dims.push_back({1, l->head_dim});
  for (int i = 0; i < 5; ++i) {
    if (st[i] < 0 || st[i] % 8 != 0) return CR_ERR_LAYOUT;
    if (ext[i] > 1) dims.push_back({st[i], ext[i]});
  }
  return check_injective(dims);
}

// ... and validity of the host block table for n_tokens tokens.
inline cr_status check_pages(const cr_kv_layout* l, const cr_kv_pages* pg, int64_t n_tokens) {
  const int bs = pg->block_size;
  const cr_status inj = check_page_strides(l, bs, pg->n_blocks, pg->stride_block);
  if (inj != CR_OK) return inj;
  const int64_t nb = (n_tokens + bs - 1) / bs;
  if (nb == 0) return CR_OK;
  if (!pg->block_table) return CR_ERR_NULL;
  std::vector<int32_t> ids(pg->block_table, pg->block_table + nb);
  for (int32_t b : ids)
    if (b < 0 || b >= pg->n_blocks) return CR_ERR_LAYOUT;
  std::sort(ids.begin(), ids.end());
  if (std::adjacent_find(ids.begin(), ids.end()) != ids.end()) return CR_ERR_LAYOUT;
  return CR_OK;
}

inline int log2_int(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Target rotary encoding: frequencies in fp64 from theta or the caller's
// table.  Returns CR_ERR_DIMS for a non-finite or non-positive field.
inline cr_status key_rope_of(const cr_rope* r, int head_dim, cr::KeyRope* kr) {
  if (!r || head_dim / 2 > 128) return CR_ERR_DIMS;
  if (!(r->scale > 0.f) || !std::isfinite(r->scale)) return CR_ERR_DIMS;
  kr->half = head_dim / 2;
  kr->scale = r->scale;
  for (int i = 0; i < kr->half; ++i) {
    double f;
    if (r->inv_freq) {
      f = r->inv_freq[i];
    } else {
      if (!(r->theta > 0.0) || !std::isfinite(r->theta)) return CR_ERR_DIMS;
      f = std::pow(r->theta, -2.0 * i / (double)head_dim);
    }
    if (!std::isfinite(f)) return CR_ERR_DIMS;
    kr->f[i] = f;
  }
  return CR_OK;
}

inline cr_status check_device() {
  static std::atomic<int> ok[64];  // per device: 0 unknown, 1 gfx950, -1 not
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return CR_ERR_DEVICE;
  const int known = dev < 64 ? ok[dev].load(std::memory_order_relaxed) : 0;
  if (known) return known > 0 ? CR_OK : CR_ERR_DEVICE;
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return CR_ERR_DEVICE;
  const bool good = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0;
  if (dev < 64) ok[dev].store(good ? 1 : -1, std::memory_order_relaxed);
  return good ? CR_OK : CR_ERR_DEVICE;
}

}  // namespace cr
