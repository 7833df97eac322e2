// Sizes at the limits of the cache's entry points, on contexts made here without a device: every call has to return before it would use
// one.  Built and run by tests/test_cache_limits.py.
#include <cstdio>

#include "hcache_internal.h"

static int failures = 0;
#define RETURNS(want, call)                                                                              \
  do {                                                                                                   \
    const hc_status s_ = (call);                                                                         \
    if (s_ != (want) || ((want) != HC_OK && !*hc_last_error())) {                                        \
      std::printf("line %d: %s -> %d, not %d: %s\n", __LINE__, #call, (int)s_, (int)(want), hc_last_error()); \
      ++failures;                                                                                        \
    }                                                                                                    \
  } while (0)

alignas(16) static char mem[4096];

static void set(hc_ctx& c, int layers, int n_q, int n_kv, int hd, int block) {
  c.desc = hc_model_desc{layers, 256, n_q, n_kv, hd, block, 4096, 2, 1e4f, 1e-5f, HC_NORM_RMS};
  c.d_kv = n_kv * hd;
  c.block_shift = 0;
  for (int b = block; b > 1; b >>= 1) c.block_shift++;
  c.layers.assign(layers, hc_layer_state{});
}

// bf16 pages of 2 GiB and more: kernels hold a page's words in 32 bits
static void large_pages() {
  int32_t* i = reinterpret_cast<int32_t*>(mem);
  const int32_t from = 0, to = 1, n = 17, page = 0;
  struct { int n_kv, hd, block; } sizes[] = {{8192, 128, 512}, {8192, 128, 4096}, {64, 128, 65536}, {1, 64, 1 << 29}};
  for (auto& z : sizes) {
    hc_ctx c;
    set(c, 1, z.n_kv, z.n_kv, z.hd, z.block);
    RETURNS(HC_OK, hc_set_kv_pool(&c, 0, mem, 1));
    RETURNS(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV, i, 2, 3, &from, &to, &n, &page, 1, nullptr));
    RETURNS(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV, i, i, 2, 3, i, nullptr));
  }
}

// The kernels take scale * log2(e), which has to be finite too.
static void large_scale() {
  int32_t* i = reinterpret_cast<int32_t*>(mem);
  hc_ctx c;
  set(c, 1, 8, 2, 128, 16);
  RETURNS(HC_OK, hc_set_kv4_pool(&c, 0, mem, 4));
  for (float scale : {2.36e38f, 3.0e38f, 3.4028234e38f})
    RETURNS(HC_EINVAL, hc_attend_kv4(&c, 0, mem, 1024, i, 1, i, i, 1, 1, 16, i, 1, scale, 0, mem, 1024, nullptr, nullptr, 0, nullptr));
}

// More rows than a call may have: its workspace and layout are refused as the call is, and the bound is that of the most there may be.
static void many_rows() {
  struct { int n_q, n_kv, total_q; } sizes[] = {{1 << 20, 8, 2048}, {64, 8, INT32_MAX}, {1 << 30, 1 << 14, INT32_MAX}, {INT32_MAX, 1, INT32_MAX}};
  for (auto& z : sizes) {
    hc_ctx c;
    set(c, 1, z.n_q, z.n_kv, 64, 16);
    int64_t bytes = -1;
    int32_t plan[4];
    RETURNS(HC_ERANGE, hc_attend_kv4_workspace(&c.desc, 1, z.total_q, z.total_q, INT32_MAX, &bytes));
    RETURNS(HC_ERANGE, hc_diag_attend_kv4(&c.desc, 1, z.total_q, z.total_q, INT32_MAX, 7, plan));
    RETURNS(HC_ERANGE, hc_attend_kv4_workspace(&c.desc, 65536, 1, 1, INT32_MAX, &bytes));
    RETURNS(HC_OK, hc_attend_kv4_workspace_bound(&c.desc, z.total_q, INT32_MAX, &bytes));
    if (bytes < 0 || bytes > 36 << 20) {
      std::printf("bound of %lld bytes\n", (long long)bytes);
      ++failures;
    }
  }
}

int main() {
  large_pages();
  many_rows();
  large_scale();
  if (failures) return 1;
  std::printf("limits ok\n");
  return 0;
}
