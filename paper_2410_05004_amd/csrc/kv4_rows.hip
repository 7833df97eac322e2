// Token rows into the 4-bit cache and back (layout: kv4.h).
#include "kv4.h"

namespace hc {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ bf16x2 as_bf16x2(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }

// Context that row t belongs to, by 16 lanes together (c: the lane's place among them): the first s with cu[s + 1] > t,
// n_seq where there is none.  Each step of the search tells 16 parts of what is left apart.
__device__ __forceinline__ int context_of(const int32_t* cu, int n_seq, int t, int c) {
  int at = 0;
  for (int left = n_seq; left > 0;) {
    const int step = (left + 15) >> 4;
    const int i = at + (c + 1) * step - 1;
    const bool behind = i < n_seq && cu[i + 1] <= t;
    const int field = (threadIdx.x & 63) & ~15;
    at += __popc((uint32_t)(__ballot(behind) >> field) & 0xffffu) * step;
    left = step > 1 ? step : 0;
  }
  return at < n_seq ? at : n_seq;
}

// A workgroup takes 16 rows; 16 lanes take 128 columns of a row, 8 values (16 bytes) a lane, and go on in steps of
// 128 * gridDim.y columns.  32 channels are four lanes: their largest magnitude is a maximum of bf16 patterns.
//   scale = smallest 2^e with top <= 7 * 2^e: with top = 1.m * 2^E, e = E - 2 if 1.m <= 1.75, else E - 1
// (then no value is further from its code than half a step, up to 7 * 2^125, where the scale ends: beyond, 6 * 2^125 is the nearest); codes by the conversion instruction, to nearest, ties to even.
// Consecutive tokens make whole sub-blocks, so a workgroup's stores fill the lines that they touch.
// Rows go past the caches, codes do not: they are what is read next, and fill lines by the store of several waves.
// Bound: memory (2 + 17 / 32 bytes a value): 32768 tokens of 8 heads of 128, 170 MB, 38 us in, 31 out (4.5 and 5.5 TB/s; a large copy: 4.9; rows
// through the caches 44 and 46), 2501 tokens of 40 heads, 65 MB, 17 and 12 (18 and 19); 64 tokens of 8 heads 3, latency.
template <Kv4Move MOVE>
__global__ __launch_bounds__(256) void kv4_rows_kernel(const Kv4RowsArgs a) {
  const int t = blockIdx.x * 16 + (threadIdx.x >> 4), c = threadIdx.x & 15;
  // lanes of rows behind the last one stay for the search's ballots and the maxima
  const bool in = t < a.n_tok;
  const int s = a.cu_seqlens ? context_of(a.cu_seqlens, a.n_seq, in ? t : a.n_tok - 1, c) : 0;
  int bad = 0, pos = 0;
  long page = 0, src_page = 0;
  if (in) {
    pos = a.positions[t];
    if (s >= a.n_seq || pos < 0 || pos >= a.max_position || (pos >> a.block_shift) >= a.max_blocks) bad = HC_DEV_BAD_POSITION;
    else {
      page = a.block_tables[(size_t)s * a.max_blocks + (pos >> a.block_shift)];
      if (page < 0 || page >= a.num_pages) bad = HC_DEV_BAD_PAGE;
      if (MOVE == Kv4Move::kPagesToCodes) {
        if ((pos >> a.block_shift) >= a.src_blocks) bad = HC_DEV_BAD_POSITION;
        else {
          src_page = a.src_table[pos >> a.block_shift];
          if (src_page < 0 || src_page >= a.src_pages) bad = HC_DEV_BAD_PAGE;
        }
      }
    }
    if (bad && c == 0 && blockIdx.y == 0) atomicOr(a.err, bad);
  }
  const bool ok = in && !bad;
  const int slot = pos & ((1 << a.block_shift) - 1);
  const int token = slot & (kSubTokens - 1), hd = a.head_dim;
  const int subs = 1 << (a.block_shift - 4);
  for (int col = (blockIdx.y * 16 + c) * 8; col < 2 * a.d_kv; col += gridDim.y * 128) {   // 2 * d_kv is a multiple of 128: no lane leaves early
    const int part = col >= a.d_kv, ch_all = col - part * a.d_kv;
    const int head = ch_all / hd, ch = ch_all - head * hd;
    uint8_t* block = a.pool + (((size_t)page * a.n_kv + head) * subs + (slot >> 4)) * sub_bytes(hd);
    const int group = ch >> 5;
    uint8_t* scale_at = part ? block + v_scales_at(hd) + ((token >> 2) * (hd >> 5) + group) * 4 + (token & 3)
                             : block + k_scales_at(hd) + token * (hd >> 5) + group;
    // of V: 8 channels are two slices of 4 (hd = 64), one of 8 (128), or half of one of 16 (256)
    const int slice = ch * 16 / hd;
    uint8_t* code_at = part ? block + v_codes_at(hd) + (((token >> 2) * 16 + slice) * 4 + (token & 3)) * (hd >> 5) + (hd == 256 ? (ch & 8) >> 1 : 0)
                            : block + token * (hd >> 1) + (ch >> 1);
    const bool halves = part && hd == 64;                 // the second slice's two bytes are four tokens' further on
    if (MOVE == Kv4Move::kCodesToRows) {
      if (!ok) continue;
      uint32_t w;
      if (halves) w = *reinterpret_cast<const uint16_t*>(code_at) | (uint32_t)*reinterpret_cast<const uint16_t*>(code_at + 8) << 16;
      else        w = *reinterpret_cast<const uint32_t*>(code_at);
      const float scale = __uint_as_float((uint32_t)*scale_at << 23);
      u32x4 out;
      out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
      out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
      out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
      out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
      __builtin_nontemporal_store(out, reinterpret_cast<u32x4*>(a.rows + (size_t)t * (2 * a.d_kv) + col));
    } else {
      u32x4 x = {0, 0, 0, 0};
      if (ok) {
        const uint16_t* src = MOVE == Kv4Move::kRowsToCodes
            ? a.rows + (size_t)t * (2 * a.d_kv) + col
            : a.src_pool + ((((size_t)src_page * 2 + part) << a.block_shift) + slot) * a.d_kv + ch_all;
        x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src));
      }
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t hi = (x[i] >> 16) & 0x7fffu, lo = x[i] & 0x7fffu;
        top = top > hi ? top : hi;
        top = top > lo ? top : lo;
      }
#pragma unroll
      for (int m = 1; m <= 2; m <<= 1) {
        const uint32_t o = __shfl_xor(top, m);
        top = top > o ? top : o;
      }
      if (!ok) continue;
      int e = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x60u ? 1 : 0);
      e = e < kMinScale ? kMinScale : e > kMaxScale ? kMaxScale : e;
      uint32_t w = 0;
      if (top >= 0x7f80u) e = kNanScale;                  // an infinity or a NaN: the group's values are lost
      else {
        const float scale = __uint_as_float((uint32_t)e << 23);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf16x2(x[0]), scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf16x2(x[1]), scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf16x2(x[2]), scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, as_bf16x2(x[3]), scale, 3);
      }
      if (halves) {
        *reinterpret_cast<uint16_t*>(code_at) = (uint16_t)w;
        *reinterpret_cast<uint16_t*>(code_at + 8) = (uint16_t)(w >> 16);
      } else {
        *reinterpret_cast<uint32_t*>(code_at) = w;
      }
      if ((c & 3) == 0) *scale_at = (uint8_t)e;
    }
  }
}

hipError_t launch_kv4_rows(const Kv4RowsArgs& a, Kv4Move move, hipStream_t stream) {
  if (a.n_tok <= 0) return hipSuccess;
  const int tiles = (a.n_tok + 15) / 16, cols = 2 * a.d_kv / 128;
  // columns go to workgroups of their own until there are some 4096 of them
  int by = tiles < 4096 ? (4096 + tiles - 1) / tiles : 1;
  if (by > cols) by = cols;
  const dim3 grid(tiles, by);
  switch (move) {
    case Kv4Move::kRowsToCodes: hipLaunchKernelGGL(kv4_rows_kernel<Kv4Move::kRowsToCodes>, grid, dim3(256), 0, stream, a); break;
    case Kv4Move::kPagesToCodes: hipLaunchKernelGGL(kv4_rows_kernel<Kv4Move::kPagesToCodes>, grid, dim3(256), 0, stream, a); break;
    case Kv4Move::kCodesToRows: hipLaunchKernelGGL(kv4_rows_kernel<Kv4Move::kCodesToRows>, grid, dim3(256), 0, stream, a); break;
  }
  return hipGetLastError();
}

}  // namespace hc
