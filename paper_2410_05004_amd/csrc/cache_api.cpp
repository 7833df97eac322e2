// Entry points of the 4-bit cache and of pages as a whole: argument validation and launches.
#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <vector>

#include "kv4.h"
#include "pages.h"

using namespace hc;

namespace {

// The context's device for the time of a call.
class OnDevice {
 public:
  explicit OnDevice(const hc_ctx* ctx) {
    err = hipGetDevice(&before_);
    if (err == hipSuccess && before_ != ctx->device) {
      err = hipSetDevice(ctx->device);
      moved_ = err == hipSuccess;
    }
  }
  ~OnDevice() {
    if (moved_) (void)hipSetDevice(before_);
  }
  hipError_t err;

 private:
  int before_ = 0;
  bool moved_ = false;
};

int64_t kv4_page_bytes(const hc_model_desc& d) {
  return (int64_t)d.n_kv_heads * (d.block_size / kSubTokens) * sub_bytes(d.head_dim);
}

hc_status check_kv4(const hc_model_desc& d) {
  if (!attend_head_dim(d.head_dim)) return fail(HC_EINVAL, "the 4-bit cache needs head_dim 64, 128 or 256");
  if (d.block_size < kSubTokens) return fail(HC_EINVAL, "the 4-bit cache needs block_size >= 16");
  if (kv4_page_bytes(d) > INT_MAX) return fail(HC_EINVAL, "a page of the 4-bit cache must stay below 2 GiB");   // kernels hold it in 32 bits
  return HC_OK;
}

hc_status check_layer4(const hc_ctx* ctx, int32_t layer) {
  const hc_status s = check_layer(ctx, layer);
  if (s != HC_OK) return s;
  if (!ctx->layers[layer].pool4) return fail(HC_ESTATE, "hc_set_kv4_pool was not called for this layer");
  return HC_OK;
}

// What launches, and the plan's 64-bit products, have room for.
hc_status check_attend_range(const hc_model_desc& d, int n_seq, int total_q) {
  if (n_seq > 65535) return fail(HC_ERANGE, "at most 65535 contexts");
  if ((int64_t)total_q * d.n_q_heads > INT_MAX) return fail(HC_ERANGE, "total_q * n_q_heads must stay below 2^31");
  return HC_OK;
}

// A window leaves fewer keys to share than the sizes say; the workspace is that of all keys.
AttendPlan plan_window(const hc_model_desc& d, const AttendPlan& all, int n_seq, int total_q, int max_q, int max_kv, int window) {
  if (window == 0) return all;
  AttendPlan plan = plan_attend(d.n_q_heads, d.n_kv_heads, d.head_dim, n_seq, total_q, max_q, (int)std::min<int64_t>(max_kv, (int64_t)window + max_q));
  plan.n_split = std::min(plan.n_split, all.n_split);
  return plan;
}

Kv4RowsArgs rows_args(const hc_ctx* ctx, int32_t layer, const int32_t* d_positions, int32_t n_tok, const int32_t* d_cu,
                      int32_t n_seq, const int32_t* d_tables, int32_t max_blocks) {
  const hc_layer_state& L = ctx->layers[layer];
  Kv4RowsArgs a{};
  a.pool = L.pool4;
  a.positions = d_positions;
  a.cu_seqlens = d_cu;
  a.block_tables = d_tables;
  a.err = ctx->err_dev;
  a.num_pages = L.num_pages4;
  a.n_seq = n_seq;
  a.max_blocks = max_blocks;
  a.n_tok = n_tok;
  a.d_kv = ctx->d_kv;
  a.head_dim = ctx->desc.head_dim;
  a.n_kv = ctx->desc.n_kv_heads;
  a.block_shift = ctx->block_shift;
  a.max_position = ctx->desc.max_position;
  return a;
}

hc_status move_rows(hc_ctx* ctx, int32_t layer, void* d_rows, const int32_t* d_positions, int32_t n_tok, const int32_t* d_cu,
                    int32_t n_seq, const int32_t* d_tables, int32_t max_blocks, Kv4Move move, void* stream) {
  clear_error();
  hc_status s = check_layer4(ctx, layer);
  if (s != HC_OK) return s;
  if (n_tok < 0 || n_seq < 0 || max_blocks < 0) return fail(HC_EINVAL, "negative size");
  if (n_tok == 0 || n_seq == 0) return HC_OK;
  if (!d_rows || !d_positions || !d_tables) return fail(HC_EINVAL, "null device pointer");
  if (!d_cu && n_seq != 1) return fail(HC_EINVAL, "several contexts need d_cu_seqlens");
  if (!aligned16(d_rows)) return fail(HC_EALIGN, "rows not 16-byte aligned");
  OnDevice on(ctx);
  HC_HIP(on.err);
  Kv4RowsArgs a = rows_args(ctx, layer, d_positions, n_tok, d_cu, n_seq, d_tables, max_blocks);
  a.rows = static_cast<uint16_t*>(d_rows);
  HC_HIP(launch_kv4_rows(a, move, static_cast<hipStream_t>(stream)));
  return HC_OK;
}

// The pools that a call on whole pages is about: every layer's, of as many pages each.
hc_status page_pools(const hc_ctx* ctx, int32_t pools, std::vector<void*>& list, int& first4, PageShape shape[2], int64_t& num_pages) {
  if (pools < 1 || pools > (HC_POOL_KV | HC_POOL_KV4)) return fail(HC_EINVAL, "pools must be HC_POOL_KV, HC_POOL_KV4 or both");
  const hc_model_desc& d = ctx->desc;
  num_pages = -1;
  for (int kind = 0; kind < 2; ++kind) {
    if (kind == 1) first4 = (int)list.size();
    if (!(pools & (kind ? HC_POOL_KV4 : HC_POOL_KV))) continue;
    for (const hc_layer_state& L : ctx->layers) {
      void* p = kind ? static_cast<void*>(L.pool4) : static_cast<void*>(L.pool);
      const int64_t n = kind ? L.num_pages4 : L.num_pages;
      if (!p) return fail(HC_ESTATE, kind ? "a layer has no 4-bit pool" : "a layer has no bf16 pool");
      if (num_pages >= 0 && n != num_pages) return fail(HC_EINVAL, "the pools differ in their number of pages");
      num_pages = n;
      list.push_back(p);
    }
  }
  const int64_t half_words = (int64_t)d.block_size * ctx->d_kv / 8;    // 16-byte words; d_kv is a multiple of 64
  if ((pools & HC_POOL_KV) && 2 * half_words * 16 > INT_MAX) return fail(HC_EINVAL, "a page of the bf16 cache must stay below 2 GiB");
  const int kv_half = pools & HC_POOL_KV ? (int)half_words : 0;
  shape[0] = PageShape{2 * kv_half, 2, kv_half, ctx->d_kv / 8, 0};
  if (pools & HC_POOL_KV4) {
    const int sub = sub_bytes(d.head_dim) / 16, head = d.block_size / kSubTokens * sub;
    shape[1] = PageShape{d.n_kv_heads * head, d.n_kv_heads, head, sub, 4};
  } else {
    shape[1] = shape[0];
  }
  return HC_OK;
}

// Pools [at, at + n) of `list` into a launch's arguments.
void some_pools(PoolList& to, const std::vector<void*>& list, int first4, const PageShape shape[2], int at) {
  const int n = std::min<int>(kPoolsPerLaunch, (int)list.size() - at);
  std::copy_n(list.begin() + at, n, to.pool);
  to.n_pools = n;
  to.first4 = std::min(std::max(first4 - at, 0), n);
  to.shape[0] = shape[0];
  to.shape[1] = shape[1];
}

bool has_twice(std::vector<int32_t> v) {
  std::sort(v.begin(), v.end());
  return std::adjacent_find(v.begin(), v.end()) != v.end();
}

hc_status fork_pages(hc_ctx* ctx, int32_t pools, int32_t* d_tables, int32_t n_rows, int32_t max_blocks, const int32_t* from,
                     const int32_t* to, const int32_t* n_tok, const int32_t* new_pages, int32_t n_fork, hipStream_t stream) {
  std::vector<void*> list;
  PageShape shape[2];
  int first4 = 0;
  int64_t num_pages = 0;
  hc_status s = page_pools(ctx, pools, list, first4, shape, num_pages);
  if (s != HC_OK) return s;
  const int block = ctx->desc.block_size;
  std::vector<int32_t> pages, targets(to, to + n_fork);
  for (int i = 0; i < n_fork; ++i) {
    if (from[i] < 0 || from[i] >= n_rows || to[i] < 0 || to[i] >= n_rows) return fail(HC_ERANGE, "fork: row outside the tables");
    if (n_tok[i] < 0 || n_tok[i] > (int64_t)max_blocks * block) return fail(HC_ERANGE, "fork: more tokens than the table has room for");
    if (n_tok[i] % block == 0) continue;
    if (new_pages[i] < 0 || new_pages[i] >= num_pages) return fail(HC_ERANGE, "fork: new page outside the pools");
    pages.push_back(new_pages[i]);
  }
  if (has_twice(pages)) return fail(HC_EINVAL, "fork: a new page is given twice");
  if (has_twice(targets)) return fail(HC_EINVAL, "fork: a row is the target of two forks");
  std::sort(targets.begin(), targets.end());
  for (int i = 0; i < n_fork; ++i)
    if (std::binary_search(targets.begin(), targets.end(), from[i])) return fail(HC_EINVAL, "fork: a row is both source and target");
  OnDevice on(ctx);
  HC_HIP(on.err);
  for (int f0 = 0; f0 < n_fork; f0 += kForksPerLaunch) {
    ForkArgs a{};
    a.n_fork = std::min(kForksPerLaunch, n_fork - f0);
    a.tables = d_tables;
    a.err = ctx->err_dev;
    a.num_pages = num_pages;
    a.max_blocks = max_blocks;
    a.block_shift = ctx->block_shift;
    int most = 0;                                            // words of a page that any fork copies
    for (int i = 0; i < a.n_fork; ++i) {
      a.from[i] = from[f0 + i];
      a.to[i] = to[f0 + i];
      a.n_tok[i] = n_tok[f0 + i];
      a.page[i] = new_pages[f0 + i];
      const int rest = a.n_tok[i] % block;
      for (int k = first4 == 0 ? 1 : 0; k < (first4 < (int)list.size() ? 2 : 1); ++k)
        most = std::max(most, shape[k].runs * ((rest + (1 << shape[k].unit_shift) - 1) >> shape[k].unit_shift) * shape[k].unit);
    }
    a.pieces = std::max(1, (most + kForkPiece - 1) / kForkPiece);
    for (int at = 0; at < (int)list.size(); at += kPoolsPerLaunch) {
      some_pools(a.pools, list, first4, shape, at);
      a.with_tables = at + kPoolsPerLaunch >= (int)list.size();
      // a pool to a workgroup until there are 4096 of them (64 forks of 17 KiB pages in 80 layers: 39 us in 1024, 33 in 4096)
      a.shares = std::max(1, std::min(std::max(a.pools.first4, a.pools.n_pools - a.pools.first4), 4096 / (a.pieces * a.n_fork)));
      HC_HIP(launch_fork(a, stream));
    }
  }
  return HC_OK;
}

hc_status compact_pages(hc_ctx* ctx, int32_t pools, const int32_t* d_in, int32_t* d_out, int32_t n_rows, int32_t max_blocks,
                        int32_t* d_plan, hipStream_t stream) {
  std::vector<void*> list;
  CompactArgs a{};
  PageShape shape[2];
  int first4 = 0;
  int64_t num_pages = 0;
  hc_status s = page_pools(ctx, pools, list, first4, shape, num_pages);
  if (s != HC_OK) return s;
  if (num_pages > kMaxCompactPages) return fail(HC_ERANGE, "hc_compact_pages takes at most 2^20 pages");
  OnDevice on(ctx);
  HC_HIP(on.err);
  a.tables_in = d_in;
  a.tables_out = d_out;
  a.plan = d_plan;
  a.err = ctx->err_dev;
  a.entries = (int64_t)n_rows * max_blocks;
  a.num_pages = (int32_t)num_pages;
  HC_HIP(launch_compact_plan(a, stream));
  for (int at = 0; at < (int)list.size(); at += kPoolsPerLaunch) {
    some_pools(a.pools, list, first4, shape, at);
    a.with_tables = at == 0;
    HC_HIP(launch_compact_move(a, stream));
  }
  return HC_OK;
}

}  // namespace

extern "C" {

hc_status hc_kv4_page_bytes(const hc_model_desc* desc, int64_t* out_bytes) {
  clear_error();
  if (!out_bytes) return fail(HC_EINVAL, "null output pointer");
  hc_status s = check_desc(desc);
  if (s == HC_OK) s = check_kv4(*desc);
  if (s != HC_OK) return s;
  *out_bytes = kv4_page_bytes(*desc);
  return HC_OK;
}

hc_status hc_set_kv4_pool(hc_ctx* ctx, int32_t layer, void* d_pool, int64_t num_pages) {
  clear_error();
  hc_status s = check_layer(ctx, layer);
  if (s == HC_OK) s = check_kv4(ctx->desc);
  if (s != HC_OK) return s;
  if (!d_pool) return fail(HC_EINVAL, "pool pointer is null");
  if (!aligned16(d_pool)) return fail(HC_EALIGN, "pool not 16-byte aligned");
  if (num_pages <= 0 || num_pages > (((int64_t)1 << 31) - 1) / (2 * ctx->desc.block_size))
    return fail(HC_ERANGE, "num_pages out of range (num_pages * 2 * block_size must stay below 2^31)");
  ctx->layers[layer].pool4 = static_cast<uint8_t*>(d_pool);
  ctx->layers[layer].num_pages4 = num_pages;
  return HC_OK;
}

hc_status hc_quantize_kv(hc_ctx* ctx, int32_t layer, const void* d_rows, const int32_t* d_positions, int32_t h_total_tokens,
                         const int32_t* d_cu_seqlens, int32_t n_seq, const int32_t* d_block_tables, int32_t max_blocks,
                         void* stream) {
  return move_rows(ctx, layer, const_cast<void*>(d_rows), d_positions, h_total_tokens, d_cu_seqlens, n_seq, d_block_tables,
                   max_blocks, Kv4Move::kRowsToCodes, stream);
}

hc_status hc_dequantize_kv(hc_ctx* ctx, int32_t layer, void* d_rows, const int32_t* d_positions, int32_t h_total_tokens,
                           const int32_t* d_cu_seqlens, int32_t n_seq, const int32_t* d_block_tables, int32_t max_blocks,
                           void* stream) {
  return move_rows(ctx, layer, d_rows, d_positions, h_total_tokens, d_cu_seqlens, n_seq, d_block_tables, max_blocks,
                   Kv4Move::kCodesToRows, stream);
}

hc_status hc_quantize_kv_pages(hc_ctx* ctx, int32_t layer, const int32_t* d_positions, int32_t n_tok,
                               const int32_t* d_block_table, int32_t n_blocks, const int32_t* d_block_table4, int32_t n_blocks4,
                               void* stream) {
  clear_error();
  hc_status s = check_layer4(ctx, layer);
  if (s != HC_OK) return s;
  const hc_layer_state& L = ctx->layers[layer];
  if (!L.pool) return fail(HC_ESTATE, "hc_set_kv_pool was not called for this layer");
  if (n_tok < 0 || n_blocks < 0 || n_blocks4 < 0) return fail(HC_EINVAL, "negative size");
  if (n_tok == 0) return HC_OK;
  if (!d_positions || !d_block_table || !d_block_table4) return fail(HC_EINVAL, "null device pointer");
  OnDevice on(ctx);
  HC_HIP(on.err);
  Kv4RowsArgs a = rows_args(ctx, layer, d_positions, n_tok, nullptr, 1, d_block_table4, n_blocks4);
  a.src_pool = L.pool;
  a.src_table = d_block_table;
  a.src_pages = L.num_pages;
  a.src_blocks = n_blocks;
  HC_HIP(launch_kv4_rows(a, Kv4Move::kPagesToCodes, static_cast<hipStream_t>(stream)));
  return HC_OK;
}

hc_status hc_attend_kv4_workspace(const hc_model_desc* desc, int32_t n_seq, int32_t h_total_q, int32_t h_max_q,
                                  int32_t h_max_kv, int64_t* out_bytes) {
  clear_error();
  if (!out_bytes) return fail(HC_EINVAL, "null output pointer");
  hc_status s = check_desc(desc);
  if (s == HC_OK) s = check_kv4(*desc);
  if (s != HC_OK) return s;
  if (n_seq < 0 || h_total_q < 0 || h_max_q < 0 || h_max_kv < 0) return fail(HC_EINVAL, "negative size");
  s = check_attend_range(*desc, n_seq, h_total_q);
  if (s != HC_OK) return s;
  *out_bytes = plan_attend(desc->n_q_heads, desc->n_kv_heads, desc->head_dim, n_seq, h_total_q, h_max_q, h_max_kv).workspace;
  return HC_OK;
}

hc_status hc_attend_kv4_workspace_bound(const hc_model_desc* desc, int32_t h_total_q, int32_t h_max_kv, int64_t* out_bytes) {
  clear_error();
  if (!out_bytes) return fail(HC_EINVAL, "null output pointer");
  hc_status s = check_desc(desc);
  if (s == HC_OK) s = check_kv4(*desc);
  if (s != HC_OK) return s;
  if (h_total_q < 0 || h_max_kv < 0) return fail(HC_EINVAL, "negative size");
  *out_bytes = attend_workspace_bound(desc->n_q_heads, desc->n_kv_heads, desc->head_dim, h_total_q, h_max_kv);
  return HC_OK;
}

hc_status hc_diag_attend_kv4(const hc_model_desc* desc, int32_t n_seq, int32_t h_total_q, int32_t h_max_q, int32_t h_max_kv,
                             int32_t window, int32_t* out_plan) {
  clear_error();
  if (!out_plan) return fail(HC_EINVAL, "null output pointer");
  hc_status s = check_desc(desc);
  if (s == HC_OK) s = check_kv4(*desc);
  if (s != HC_OK) return s;
  if (n_seq < 0 || h_total_q < 0 || h_max_q < 0 || h_max_kv < 0 || window < 0) return fail(HC_EINVAL, "negative size");
  s = check_attend_range(*desc, n_seq, h_total_q);
  if (s != HC_OK) return s;
  const AttendPlan all = plan_attend(desc->n_q_heads, desc->n_kv_heads, desc->head_dim, n_seq, h_total_q, h_max_q, h_max_kv);
  const AttendPlan plan = plan_window(*desc, all, n_seq, h_total_q, h_max_q, h_max_kv, window);
  out_plan[0] = 16 * plan.row_blocks;
  out_plan[1] = plan.flat;
  out_plan[2] = plan.n_split;
  out_plan[3] = plan.paired;
  return HC_OK;
}

hc_status hc_attend_kv4(hc_ctx* ctx, int32_t layer, const void* d_q, int64_t q_stride, const int32_t* d_positions,
                        int32_t h_total_q, const int32_t* d_cu_q, const int32_t* d_kv_lens, int32_t n_seq, int32_t h_max_q,
                        int32_t h_max_kv, const int32_t* d_block_tables, int32_t max_blocks, float scale, int32_t window,
                        void* d_out, int64_t out_stride, float* d_lse, void* d_workspace, int64_t workspace_bytes,
                        void* stream) {
  clear_error();
  hc_status s = check_layer4(ctx, layer);
  if (s != HC_OK) return s;
  const hc_model_desc& d = ctx->desc;
  if (h_total_q < 0 || n_seq < 0 || h_max_q < 0 || h_max_kv < 0 || max_blocks < 0 || window < 0 || workspace_bytes < 0)
    return fail(HC_EINVAL, "negative size");
  const float scale_log2 = scale * 1.44269504089f;
  if (!(scale > 0.f) || !std::isfinite(scale_log2)) return fail(HC_EINVAL, "scale must be positive, and finite times log2(e)");
  if (h_total_q == 0 || n_seq == 0) return HC_OK;
  if (!d_q || !d_positions || !d_cu_q || !d_kv_lens || !d_block_tables || !d_out) return fail(HC_EINVAL, "null device pointer");
  const int64_t width = (int64_t)d.n_q_heads * d.head_dim;
  if (q_stride < width || q_stride % 8 || out_stride < width || out_stride % 8)
    return fail(HC_EINVAL, "strides must be multiples of 8 of at least n_q_heads * head_dim");
  if (!aligned16(d_q) || !aligned16(d_out)) return fail(HC_EALIGN, "queries or output not 16-byte aligned");
  s = check_attend_range(d, n_seq, h_total_q);
  if (s != HC_OK) return s;
  AttendPlan plan = plan_attend(d.n_q_heads, d.n_kv_heads, d.head_dim, n_seq, h_total_q, h_max_q, h_max_kv);
  if (plan.workspace) {
    if (!d_workspace || workspace_bytes < plan.workspace) return fail(HC_EINVAL, "workspace smaller than hc_attend_kv4_workspace says");
    if (!aligned16(d_workspace)) return fail(HC_EALIGN, "workspace not 16-byte aligned");
  }
  plan = plan_window(d, plan, n_seq, h_total_q, h_max_q, h_max_kv, window);
  OnDevice on(ctx);
  HC_HIP(on.err);
  const hc_layer_state& L = ctx->layers[layer];
  AttendArgs a{};
  a.q = static_cast<const uint16_t*>(d_q);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.positions = d_positions;
  a.cu_q = d_cu_q;
  a.kv_lens = d_kv_lens;
  a.block_tables = d_block_tables;
  a.pool = L.pool4;
  a.out = static_cast<uint16_t*>(d_out);
  a.lse = d_lse;
  a.part = static_cast<float*>(d_workspace);
  a.err = ctx->err_dev;
  a.num_pages = L.num_pages4;
  a.n_seq = n_seq;
  a.total_q = h_total_q;
  a.max_blocks = max_blocks;
  a.block_shift = ctx->block_shift;
  a.n_q = d.n_q_heads;
  a.n_kv = d.n_kv_heads;
  a.group = d.n_q_heads / d.n_kv_heads;
  a.window = window;
  a.scale_log2 = scale_log2;
  a.flat = plan.flat;
  a.n_slots = plan.n_slots;
  a.n_split = plan.n_split;
  HC_HIP(launch_attend(a, d.head_dim, plan, static_cast<hipStream_t>(stream)));
  return HC_OK;
}

hc_status hc_fork_pages(hc_ctx* ctx, int32_t pools, int32_t* d_block_tables, int32_t n_rows, int32_t max_blocks,
                        const int32_t* h_from_rows, const int32_t* h_to_rows, const int32_t* h_n_tok,
                        const int32_t* h_new_pages, int32_t n_fork, void* stream) {
  clear_error();
  if (!ctx) return fail(HC_EINVAL, "ctx is null");
  if (n_rows < 0 || max_blocks < 0 || n_fork < 0) return fail(HC_EINVAL, "negative size");
  if (n_fork > 0 && (!d_block_tables || !h_from_rows || !h_to_rows || !h_n_tok || !h_new_pages)) return fail(HC_EINVAL, "null pointer");
  try {
    return fork_pages(ctx, pools, d_block_tables, n_rows, max_blocks, h_from_rows, h_to_rows, h_n_tok, h_new_pages, n_fork,
                      static_cast<hipStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return fail(HC_ENOMEM, "out of host memory");
  }
}

hc_status hc_compact_pages(hc_ctx* ctx, int32_t pools, const int32_t* d_tables_in, int32_t* d_tables_out, int32_t n_rows,
                           int32_t max_blocks, int32_t* d_plan, void* stream) {
  clear_error();
  if (!ctx) return fail(HC_EINVAL, "ctx is null");
  if (n_rows < 0 || max_blocks < 0) return fail(HC_EINVAL, "negative size");
  if (!d_plan || ((n_rows && max_blocks) && (!d_tables_in || !d_tables_out))) return fail(HC_EINVAL, "null pointer");
  try {
    return compact_pages(ctx, pools, d_tables_in, d_tables_out, n_rows, max_blocks, d_plan, static_cast<hipStream_t>(stream));
  } catch (const std::bad_alloc&) {
    return fail(HC_ENOMEM, "out of host memory");
  }
}

}  // extern "C"
