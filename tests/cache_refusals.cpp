// Refusals of the entry points of the 4-bit cache and of pages as a whole.  The context is made here, without a device: every call
// has to return before it would use one.  Built and run by tests/test_kv4_oracle.py.
#include <cstdio>
#include <cstring>

#include "hcache_internal.h"

static int failures = 0;
#define REFUSED(want, call)                                                                              \
  do {                                                                                                   \
    const hc_status s_ = (call);                                                                         \
    if (s_ != (want) || ((want) != HC_OK && !*hc_last_error())) {                                        \
      std::printf("line %d: %s -> %d, not %d: %s\n", __LINE__, #call, (int)s_, (int)(want), hc_last_error()); \
      ++failures;                                                                                        \
    }                                                                                                    \
  } while (0)

alignas(16) static char mem[4096];

static void set(hc_ctx& c, int layers, int hd, int block) {
  c.desc = hc_model_desc{layers, 256, 8, 2, hd, block, 4096, 2, 1e4f, 1e-5f, HC_NORM_RMS};
  c.d_kv = 2 * hd;
  c.block_shift = 0;
  for (int b = block; b > 1; b >>= 1) c.block_shift++;
  c.layers.assign(layers, hc_layer_state{});
}

int main() {
  hc_ctx c;
  set(c, 2, 128, 16);
  int32_t* i = reinterpret_cast<int32_t*>(mem);
  float* f = reinterpret_cast<float*>(mem);
  char* odd = mem + 2;
  // ---- pools
  hc_ctx narrow, small;
  set(narrow, 1, 192, 16);
  set(small, 1, 128, 8);
  REFUSED(HC_EINVAL, hc_set_kv4_pool(&narrow, 0, mem, 4));
  REFUSED(HC_EINVAL, hc_set_kv4_pool(&small, 0, mem, 4));
  REFUSED(HC_ERANGE, hc_set_kv4_pool(&c, 2, mem, 4));
  REFUSED(HC_ERANGE, hc_set_kv4_pool(&c, -1, mem, 4));
  REFUSED(HC_EINVAL, hc_set_kv4_pool(&c, 0, nullptr, 4));
  REFUSED(HC_EALIGN, hc_set_kv4_pool(&c, 0, odd, 4));
  REFUSED(HC_ERANGE, hc_set_kv4_pool(&c, 0, mem, 0));
  REFUSED(HC_ERANGE, hc_set_kv4_pool(&c, 0, mem, INT64_MAX));
  // ---- out of order
  REFUSED(HC_ESTATE, hc_quantize_kv(&c, 0, mem, i, 1, i, 1, i, 1, nullptr));
  REFUSED(HC_ESTATE, hc_dequantize_kv(&c, 0, mem, i, 1, i, 1, i, 1, nullptr));
  REFUSED(HC_ESTATE, hc_quantize_kv_pages(&c, 0, i, 1, i, 1, i, 1, nullptr));
  REFUSED(HC_ESTATE, hc_attend_kv4(&c, 0, mem, 1024, i, 1, i, i, 1, 1, 1, i, 1, 1.f, 0, mem, 1024, f, nullptr, 0, nullptr));
  REFUSED(HC_OK, hc_set_kv4_pool(&c, 0, mem, 4));
  REFUSED(HC_ESTATE, hc_quantize_kv_pages(&c, 0, i, 1, i, 1, i, 1, nullptr));      // no bf16 pool
  REFUSED(HC_ESTATE, hc_fork_pages(&c, HC_POOL_KV4, i, 4, 4, i, i, i, i, 1, nullptr));   // layer 1 has none
  REFUSED(HC_ESTATE, hc_compact_pages(&c, HC_POOL_KV4, i, i, 4, 4, i, nullptr));
  REFUSED(HC_OK, hc_set_kv4_pool(&c, 1, mem, 4));
  REFUSED(HC_ESTATE, hc_compact_pages(&c, HC_POOL_KV4 | HC_POOL_KV, i, i, 4, 4, i, nullptr));
  REFUSED(HC_OK, hc_set_kv_pool(&c, 0, mem, 4));
  REFUSED(HC_OK, hc_set_kv_pool(&c, 1, mem, 5));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV, i, i, 4, 4, i, nullptr));    // 4 and 5 pages
  // ---- rows
  for (auto fn : {+[](hc_ctx* x, int l, char* r, int32_t* p, int n, int32_t* cu, int s, int32_t* t, int b) { return hc_quantize_kv(x, l, r, p, n, cu, s, t, b, nullptr); },
                  +[](hc_ctx* x, int l, char* r, int32_t* p, int n, int32_t* cu, int s, int32_t* t, int b) { return hc_dequantize_kv(x, l, r, p, n, cu, s, t, b, nullptr); }}) {
    REFUSED(HC_ERANGE, fn(&c, 2, mem, i, 1, i, 1, i, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, i, -1, i, 1, i, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, i, 1, i, -1, i, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, i, 1, i, 1, i, -1));
    REFUSED(HC_EINVAL, fn(&c, 0, nullptr, i, 1, i, 1, i, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, nullptr, 1, i, 1, i, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, i, 1, i, 1, nullptr, 1));
    REFUSED(HC_EINVAL, fn(&c, 0, mem, i, 1, nullptr, 2, i, 1));
    REFUSED(HC_EALIGN, fn(&c, 0, odd, i, 1, i, 1, i, 1));
    REFUSED(HC_OK, fn(&c, 0, nullptr, nullptr, 0, nullptr, 1, nullptr, 1));
    REFUSED(HC_OK, fn(&c, 0, mem, i, 1, i, 0, i, 1));
  }
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, i, -1, i, 1, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, i, 1, i, -1, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, i, 1, i, 1, i, -1, nullptr));
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, nullptr, 1, i, 1, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, i, 1, nullptr, 1, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_quantize_kv_pages(&c, 0, i, 1, i, 1, nullptr, 1, nullptr));
  REFUSED(HC_OK, hc_quantize_kv_pages(&c, 0, nullptr, 0, nullptr, 1, nullptr, 1, nullptr));
  // ---- attention
  struct Call {
    int layer = 0;
    const void* q = mem;
    int64_t qs = 1024;
    const int32_t *p, *cu, *len, *t;
    int n = 1, seqs = 1, mq = 1, mk = 16, blocks = 1, window = 0;
    float scale = 1.f;
    void* out = mem;
    int64_t os = 1024;
    void* ws = nullptr;
    int64_t wb = 0;
  } d;
  d.p = d.cu = d.len = d.t = i;
  auto attend = [&](const Call& x) {
    return hc_attend_kv4(&c, x.layer, x.q, x.qs, x.p, x.n, x.cu, x.len, x.seqs, x.mq, x.mk, x.t, x.blocks, x.scale, x.window, x.out, x.os, f,
                         x.ws, x.wb, nullptr);
  };
#define BAD(want, field, value)  \
  do {                           \
    Call x = d;                  \
    x.field = value;             \
    REFUSED(want, attend(x));    \
  } while (0)
  BAD(HC_ERANGE, layer, 2);
  BAD(HC_EINVAL, q, nullptr);
  BAD(HC_EALIGN, q, odd);
  BAD(HC_EINVAL, qs, 1016);
  BAD(HC_EINVAL, qs, 1028);
  BAD(HC_EINVAL, os, 1016);
  BAD(HC_EINVAL, os, 1028);
  BAD(HC_EINVAL, p, nullptr);
  BAD(HC_EINVAL, cu, nullptr);
  BAD(HC_EINVAL, len, nullptr);
  BAD(HC_EINVAL, t, nullptr);
  BAD(HC_EINVAL, out, nullptr);
  BAD(HC_EALIGN, out, odd);
  BAD(HC_EINVAL, n, -1);
  BAD(HC_EINVAL, seqs, -1);
  BAD(HC_EINVAL, mq, -1);
  BAD(HC_EINVAL, mk, -1);
  BAD(HC_EINVAL, blocks, -1);
  BAD(HC_EINVAL, window, -1);
  BAD(HC_EINVAL, scale, 0.f);
  BAD(HC_EINVAL, scale, -1.f);
  BAD(HC_EINVAL, scale, __builtin_nanf(""));
  BAD(HC_EINVAL, scale, __builtin_inff());
  BAD(HC_EINVAL, wb, -1);
  BAD(HC_ERANGE, seqs, 65536);
  BAD(HC_ERANGE, n, 1 << 28);
  BAD(HC_OK, n, 0);
  BAD(HC_OK, seqs, 0);
  int64_t need = 0;
  REFUSED(HC_OK, hc_attend_kv4_workspace(&c.desc, 1, 1, 1, 100000, &need));
  d.mk = 100000;
  BAD(HC_EINVAL, ws, nullptr);
  d.ws = mem;
  BAD(HC_EINVAL, wb, need - 1);
  d.ws = odd;
  BAD(HC_EALIGN, wb, need);
  REFUSED(HC_EINVAL, hc_attend_kv4_workspace(&c.desc, 1, 1, 1, 1, nullptr));
  // ---- fork: two layers of 4 pages
  auto fork = [&](int pools, std::vector<int32_t> from, std::vector<int32_t> to, std::vector<int32_t> n, std::vector<int32_t> page) {
    return hc_fork_pages(&c, pools, i, 5, 3, from.data(), to.data(), n.data(), page.data(), (int)from.size(), nullptr);
  };
  REFUSED(HC_EINVAL, fork(0, {0}, {1}, {17}, {3}));
  REFUSED(HC_EINVAL, fork(4, {0}, {1}, {17}, {3}));
  REFUSED(HC_EINVAL, fork(HC_POOL_KV, {0}, {1}, {17}, {3}));           // 4 and 5 pages
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {5}, {1}, {17}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {-1}, {1}, {17}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {5}, {17}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {-1}, {17}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {1}, {-1}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {1}, {49}, {3}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {1}, {17}, {4}));
  REFUSED(HC_ERANGE, fork(HC_POOL_KV4, {0}, {1}, {17}, {-1}));
  REFUSED(HC_EINVAL, fork(HC_POOL_KV4, {0, 0}, {1, 2}, {17, 18}, {3, 3}));
  REFUSED(HC_EINVAL, fork(HC_POOL_KV4, {0, 2}, {1, 1}, {17, 18}, {3, 2}));
  REFUSED(HC_EINVAL, fork(HC_POOL_KV4, {0, 1}, {1, 2}, {17, 18}, {3, 2}));
  REFUSED(HC_EINVAL, fork(HC_POOL_KV4, {1}, {1}, {17}, {3}));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, nullptr, 5, 3, i, i, i, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, 3, nullptr, i, i, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, 3, i, nullptr, i, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, 3, i, i, nullptr, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, 3, i, i, i, nullptr, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, -1, 3, i, i, i, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, -1, i, i, i, i, 1, nullptr));
  REFUSED(HC_EINVAL, hc_fork_pages(&c, HC_POOL_KV4, i, 5, 3, i, i, i, i, -1, nullptr));
  // ---- compact
  REFUSED(HC_EINVAL, hc_compact_pages(&c, 0, i, i, 5, 3, i, nullptr));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV4, nullptr, i, 5, 3, i, nullptr));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV4, i, nullptr, 5, 3, i, nullptr));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV4, i, i, 5, 3, nullptr, nullptr));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV4, i, i, -5, 3, i, nullptr));
  REFUSED(HC_EINVAL, hc_compact_pages(&c, HC_POOL_KV4, i, i, 5, -3, i, nullptr));
  for (int l = 0; l < 2; ++l) REFUSED(HC_OK, hc_set_kv4_pool(&c, l, mem, (1 << 20) + 1));
  REFUSED(HC_ERANGE, hc_compact_pages(&c, HC_POOL_KV4, i, i, 5, 3, i, nullptr));
  if (failures) return 1;
  std::printf("refusals ok\n");
  return 0;
}
