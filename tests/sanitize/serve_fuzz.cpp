// Host-side fuzz of cr_append_kv, cr_attend and cr_attend_workspace_bytes,
// built like abi_fuzz.cpp: fake device addresses that are never dereferenced,
// host arrays on the heap with exactly the elements a call may read.  Valid
// calls end at the device check (no GPU), invalid ones at their error.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "cacherepair.h"

static std::mt19937_64 rng(20260917);
// The first value is the common, valid choice (taken 15 times in 16).
static int64_t pick(std::initializer_list<int64_t> v) {
  if (rng() % 16 != 0) return *v.begin();
  return *(v.begin() + rng() % v.size());
}
static int64_t any(std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); }
static int counts[16];
static void tally(cr_status s) { counts[-s < 16 && s <= 0 ? -s : 15]++; }
static void* device(int i) { return reinterpret_cast<void*>(uintptr_t(i) << 40); }

int main(int argc, char** argv) {
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) == hipSuccess && n_dev > 0) {
    std::printf("serve_fuzz: a GPU is visible; this host-only check does not run there\n");
    return 0;
  }
  const long iters = argc > 1 ? std::atol(argv[1]) : 20000;
  for (long it = 0; it < iters; ++it) {
    cr_kv_layout l;
    l.n_layers = (int32_t)pick({2, 1, 36, 0, -1});
    l.n_kv_heads = (int32_t)pick({any({1, 2, 8}), 0, -2, 1 << 20});
    l.head_dim = (int32_t)pick({any({32, 64, 96, 128, 256}), 16, 512, 0});
    l.dtype = (int32_t)pick({any({CR_DTYPE_BF16, CR_DTYPE_F32}), 7, -1});
    const int64_t row = (int64_t)l.n_kv_heads * l.head_dim;
    cr_sequences q{};
    q.n_seqs = (int32_t)pick({any({1, 3, 700}), 0, -1});
    q.block_size = (int32_t)pick({any({16, 1, 1024}), 3, 0, -16, 2048});
    q.n_blocks = (int32_t)pick({100, 1, 0, INT32_MAX});
    q.max_blocks = (int32_t)pick({any({1, 9, 4096}), 0, -1, INT32_MAX});
    q.kv_lens = static_cast<int32_t*>(pick({1, 0}) ? device(1) : nullptr);
    q.block_table = static_cast<int32_t*>(pick({1, 0}) ? device(2) : nullptr);
    q.stride_block = pick({q.block_size * row, 8, -8, 12, INT64_MAX - 7, (int64_t)1 << 55});
    l.stride_head = pick({l.head_dim, l.head_dim + 16, 0, -8, 12});
    l.stride_token = pick({row, row + 64, 8, -16, (int64_t)1 << 62});
    l.stride_kv = pick({(int64_t)q.n_blocks * q.block_size * row, 8, INT64_MAX - 7});
    l.stride_layer = pick({l.stride_kv < (int64_t)1 << 60 ? 2 * l.stride_kv : 16, 16, INT64_MIN + 8});
    const int n = q.n_seqs > 0 ? q.n_seqs + 1 : 1;
    int32_t* off = new int32_t[n];
    off[0] = (int32_t)pick({0, 1});
    const int64_t step = any({0, 1, 5, 900});
    for (int i = 1; i < n; ++i) off[i] = off[i - 1] + (int32_t)(rng() % (step + 1));
    if (n > 2 && rng() % 16 == 0) off[1] = (int32_t)any({off[2] + 1, INT32_MAX, INT32_MIN});
    if (rng() % 4) q.query_offsets = off;
    auto rows = [&](int i, int64_t heads) {
      const int64_t d = l.head_dim;
      return cr_rows{pick({1, 0}) ? static_cast<char*>(device(i)) + pick({0, 8, 32}) : nullptr,
                     pick({heads * d, 0, -8, 12, INT64_MAX - 7, (int64_t)1 << 45}), pick({d, 0, d + 8, 4})};
    };
    const int32_t heads = (int32_t)pick({any({1, 5}) * (l.n_kv_heads > 0 ? l.n_kv_heads : 1) % 1000, 0, -1, 3, 4096});
    const cr_rows k = rows(3, l.n_kv_heads), v = rows(4, l.n_kv_heads), a = rows(5, heads), o = rows(6, heads);
    const int half = l.head_dim > 0 && l.head_dim <= 512 ? l.head_dim / 2 : 1;
    float* freq = new float[half];
    for (int i = 0; i < half; ++i) freq[i] = 1.f / (1 + i);
    const cr_rope rope{(double)pick({10000, 0, -1}), rng() % 2 ? freq : nullptr, rng() % 16 ? 1.0f : -1.0f};
    const int layer = (int)pick({0, 1, -1, 99});
    const bool with_q = rng() % 2;
    tally(cr_append_kv(device(7), &l, layer, &q, &k, &v, with_q ? &a : nullptr,
                       with_q != (rng() % 32 == 0) ? &o : nullptr, heads, rng() % 4 ? &rope : nullptr,
                       nullptr, nullptr));
    float* slopes = new float[heads > 0 ? heads : 1];
    for (int i = 0; i < heads; ++i) slopes[i] = 0.1f * i;
    cr_attend_options opt{};
    opt.scale = (float)pick({0, 1, -1});
    opt.softcap = (float)pick({any({0, 30}), -1});
    opt.slopes = rng() % 2 ? slopes : nullptr;
    opt.shared_len = (int32_t)pick({any({0, 1}), 5, 100000, -1, INT32_MAX});
    uint64_t bytes = 0;
    tally(cr_attend_workspace_bytes(&l, &q, heads, opt.shared_len, &bytes));
    const uint64_t given = pick({(int64_t)bytes, (int64_t)bytes - 1, 0});
    tally(cr_attend(device(7), &l, layer, &q, &a, &o, heads, rng() % 8 ? &opt : nullptr,
                    pick({1, 0}) ? device(8) : nullptr, rng() % 8 ? given : UINT64_MAX, nullptr));
    delete[] off;
    delete[] freq;
    delete[] slopes;
  }
  std::printf("serve_fuzz: %ld iterations; status counts:", iters);
  for (int i = 0; i < 16; ++i) std::printf(" %d:%d", -i, counts[i]);
  std::printf("\n");
  return 0;
}
