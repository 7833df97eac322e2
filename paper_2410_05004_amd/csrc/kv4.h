// The 4-bit KV cache: its layout, and what the translation units that read and write it share.
#pragma once

#include "hcache_internal.h"

namespace hc {

// Of 16 consecutive tokens (a sub-block of a page) a KV head's 17 * head_dim bytes are, hd = head_dim:
//   K codes   8 * hd   [token][channel / 2], the even channel in the low four bits
//   V codes   8 * hd   [token / 4][r][token % 4][hd / 32 bytes]: channels r * hd / 16 .. of 16 slices r
//   K scales  hd / 2   [token][group of 32 channels]
//   V scales  hd / 2   [token / 4][group][token % 4]
// A code is a 4-bit float (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6), a scale the
// biased exponent of a power of two, as in an fp32; 255 stands for NaN.
// The orders are those in which lane l16 of quarter q4 of a wave feeds v_mfma_f32_16x16x32: as the rows of K it takes
// token l16, channels q4 * hd / 4 .. (hd / 4 of them, in steps of 8); as the rows of V^T the channels of slice l16 and
// tokens 4 * q4 .. + 3.  Either is hd / 8 consecutive bytes, and the lanes' bytes lie side by side.
constexpr int kSubTokens = 16;
__host__ __device__ constexpr int sub_bytes(int hd) { return 17 * hd; }
__host__ __device__ constexpr int v_codes_at(int hd) { return 8 * hd; }
__host__ __device__ constexpr int k_scales_at(int hd) { return 16 * hd; }
__host__ __device__ constexpr int v_scales_at(int hd) { return 16 * hd + hd / 2; }

constexpr int kMinScale = 2, kMaxScale = 252, kNanScale = 255;   // 2^-125 and 2^125: values and products stay normal and finite

// Token rows against pages of the 4-bit pool.
struct Kv4RowsArgs {
  uint16_t* rows;              // bf16 [n_tok][K row | V row], or null: bf16 pages (src_*) are the source
  const uint16_t* src_pool;    // bf16 pool
  const int32_t* src_table;
  uint8_t* pool;
  const int32_t* positions;
  const int32_t* cu_seqlens;   // null: one context
  const int32_t* block_tables; // [n_seq][max_blocks]
  int32_t* err;
  int64_t num_pages, src_pages;
  int32_t n_seq, max_blocks, src_blocks;
  int32_t n_tok, d_kv, head_dim, n_kv, block_shift, max_position;
};
enum class Kv4Move { kRowsToCodes, kPagesToCodes, kCodesToRows };
hipError_t launch_kv4_rows(const Kv4RowsArgs& a, Kv4Move move, hipStream_t stream);

// Attention over the 4-bit pool.
constexpr int64_t kMaxKeys = 1 << 30;       // of a context: keys and what is added to them stay within 32 bits
struct AttendArgs {
  const uint16_t* q;
  int64_t q_stride, out_stride;            // elements from one token to the next
  const int32_t* positions;
  const int32_t* cu_q;
  const int32_t* kv_lens;
  const int32_t* block_tables;
  const uint8_t* pool;
  uint16_t* out;
  float* lse;                              // null: not wanted
  float* part;                             // n_split > 1: [split][row][head_dim], then [split][row][2]
  int32_t* err;
  int64_t num_pages;
  int32_t n_seq, total_q, max_blocks, block_shift;
  int32_t n_q, n_kv, group;                // query heads, KV heads, query heads of one KV head
  int32_t window;                          // 0: none
  float scale_log2;                        // softmax scale * log2(e)
  int32_t flat, n_slots, n_split;          // see AttendPlan
};
struct AttendPlan {
  int32_t row_blocks;                      // blocks of 16 rows of a workgroup; kv4_prompt.hip from 8 on
  // Places for workgroups along the rows, of a KV head and share of the keys: one a context, which goes through all of its tiles of rows
  // (one, if the sizes are right); or, flat, one a tile: context s has those from cu[s] * group / size + s on, up to one too many.
  int32_t flat, n_slots, n_split;
  bool paired;                             // contexts have up to kPairedRows rows, whose weights are kept in two parts of bf16
  int64_t workspace;                       // bytes
};
constexpr int kPairedRows = 8;             // half of a block
AttendPlan plan_attend(int n_q, int n_kv, int head_dim, int n_seq, int total_q, int max_q, int max_kv);
int64_t attend_workspace_bound(int n_q, int n_kv, int head_dim, int total_q, int max_kv);
bool attend_head_dim(int head_dim);
int attend_rows_blocks(int head_dim);      // row blocks of a workgroup of launch_attend_rows, which takes heads of 64 and 128
inline dim3 attend_grid(const AttendArgs& a) {      // places over two dimensions of less than 65536
  const int y = a.n_slots < 32768 ? a.n_slots : 32768;
  return dim3(a.n_split * a.n_kv, y, (a.n_slots + y - 1) / y);
}
void launch_attend_rows(const AttendArgs& a, int head_dim, hipStream_t stream);
hipError_t launch_attend(const AttendArgs& a, int head_dim, const AttendPlan& plan, hipStream_t stream);

}  // namespace hc
