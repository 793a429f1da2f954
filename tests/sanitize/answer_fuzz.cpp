// Host-side fuzz of cr_weigh_keys, cr_weigh_workspace_bytes, cr_choose_slots,
// cr_compact_kv and cr_sample, built like serve_fuzz.cpp: fake device addresses
// that are never dereferenced, host arrays on the heap with exactly the elements
// a call may read.
#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "cacherepair.h"

static std::mt19937_64 rng(20260921);
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
    std::printf("answer_fuzz: a GPU is visible; this host-only check does not run there\n");
    return 0;
  }
  const long iters = argc > 1 ? std::atol(argv[1]) : 20000;
  for (long it = 0; it < iters; ++it) {
    cr_kv_layout l;
    l.n_layers = (int32_t)pick({2, 1, 36, 0, -1, INT32_MAX});
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
    l.stride_kv = pick({(int64_t)(q.n_blocks < 1000 ? q.n_blocks : 1000) * q.block_size * row, 8, INT64_MAX - 7});
    l.stride_layer = pick({l.stride_kv < (int64_t)1 << 60 ? 2 * l.stride_kv : 16, 16, INT64_MIN + 8});
    const int n = q.n_seqs > 0 ? q.n_seqs + 1 : 1;
    int32_t* off = new int32_t[n];
    off[0] = (int32_t)pick({0, 1});
    const int64_t step = any({0, 1, 5, 900});
    for (int i = 1; i < n; ++i) off[i] = off[i - 1] + (int32_t)(rng() % (step + 1));
    if (n > 2 && rng() % 16 == 0) off[1] = (int32_t)any({off[2] + 1, INT32_MAX, INT32_MIN});
    if (rng() % 4) q.query_offsets = off;
    const int32_t heads = (int32_t)pick({any({1, 5}) * (l.n_kv_heads > 0 ? l.n_kv_heads : 1) % 1000, 0, -1, 3, 4096});
    const cr_rows a{pick({1, 0}) ? static_cast<char*>(device(5)) + pick({0, 8, 32}) : nullptr,
                    pick({(int64_t)heads * l.head_dim, 0, -8, 12, INT64_MAX - 7, (int64_t)1 << 45}),
                    pick({l.head_dim, 0, 4})};
    float* slopes = new float[heads > 0 ? heads : 1];
    for (int i = 0; i < heads; ++i) slopes[i] = 0.1f * i;
    cr_attend_options opt{};
    opt.scale = (float)pick({0, 1, -1});
    opt.softcap = (float)pick({any({0, 30}), -1});
    opt.slopes = rng() % 2 ? slopes : nullptr;
    opt.shared_len = (int32_t)pick({0, 5, -1});
    opt.lse = static_cast<float*>(pick({1, 0}) ? device(6) : nullptr);
    const int64_t slots = (int64_t)q.max_blocks * q.block_size;
    cr_key_weights w;
    w.data = reinterpret_cast<float*>(pick({1, 0}) ? static_cast<char*>(device(9)) + pick({0, 4, 2}) : nullptr);
    w.stride_head = pick({slots, slots + 3, 0, -4, INT64_MAX});
    w.stride_seq = pick({slots < (int64_t)1 << 40 ? (slots + 3) * (int64_t)(l.n_kv_heads > 0 ? l.n_kv_heads : 1) : 1, 1, INT64_MAX});
    w.stride_layer = pick({w.stride_seq < (int64_t)1 << 45 ? w.stride_seq * (q.n_seqs > 0 ? q.n_seqs : 1) : 1, 0, -1});
    uint64_t bytes = 0;
    tally(cr_weigh_workspace_bytes(&l, &q, heads, &bytes));
    const uint64_t given = pick({(int64_t)bytes, (int64_t)bytes - 1, 0});
    tally(cr_weigh_keys(device(7), &l, (int)pick({0, 1, -1, 99}), &q, &a, heads, rng() % 16 ? &opt : nullptr, &w,
                        pick({1, 0}) ? device(8) : nullptr, rng() % 8 ? given : UINT64_MAX, nullptr));
    cr_choice c{(int32_t)pick({any({1, 100, INT32_MAX}), 0, -1}), (int32_t)pick({any({0, 4, INT32_MAX}), -1}),
                (int32_t)pick({any({0, 64, INT32_MAX}), -1}), nullptr};
    int32_t* kept = static_cast<int32_t*>(pick({1, 0}) ? device(10) : nullptr);
    tally(cr_choose_slots(&l, &q, &w, &c, kept, static_cast<int32_t*>(device(11)), nullptr));
    int32_t* out = rng() % 2 ? static_cast<int32_t*>(device(12)) : nullptr;
    tally(cr_compact_kv(device(7), &l, &q, kept, c.budget, static_cast<int32_t*>(device(11)), out,
                        (int32_t)pick({any({1, 64}), 0, INT32_MAX}), rng() % 2 ? &w : nullptr, nullptr));
    const cr_logits x{pick({1, 0}) ? static_cast<char*>(device(13)) + pick({0, 2, 1}) : nullptr,
                      (int32_t)pick({any({CR_DTYPE_BF16, CR_DTYPE_F32}), 9}), (int32_t)pick({any({0, 1, 256}), -1, INT32_MAX}),
                      (int32_t)pick({any({1, 1000, 1 << 19}), 0, INT32_MAX}), pick({1000, 0, -1, INT64_MAX})};
    const cr_sampling o{1.f, 1.f, 0.f, 0, nullptr, nullptr, nullptr, nullptr};
    tally(cr_sample(&x, rng() % 2 ? &o : nullptr, static_cast<float*>(pick({1, 0}) ? device(14) : nullptr),
                    static_cast<int32_t*>(device(15)), nullptr, nullptr));
    delete[] off;
    delete[] slopes;
  }
  std::printf("answer_fuzz: %ld iterations; status counts:", iters);
  for (int i = 0; i < 16; ++i) std::printf(" %d:%d", -i, counts[i]);
  std::printf("\n");
  return 0;
}
