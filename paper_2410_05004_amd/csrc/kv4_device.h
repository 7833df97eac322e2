// Device helpers of the kernels that attend to the 4-bit cache.
#pragma once

#include <type_traits>

#include "kv4.h"

namespace hc {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float kNegInf = -__builtin_inff();
// The running top follows a row's maximum only when that has grown by more than this (of base 2): weights then reach
// 2^8 instead of 1, which costs nothing in floating point, and most steps rescale nothing.
constexpr float kTopSlack = 8.f;

// NaN if either is: one instruction for two of these, where fmaxf first makes every operand quiet.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

__device__ __forceinline__ uint32_t decode2(uint32_t w, float scale, int byte) {
  switch (byte) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  }
}

// The conversion reads the exponent field of its scale alone: what else the shifted word holds does no harm
// (checked for every exponent, with the other bits zero, one and mixed).
__device__ __forceinline__ float scale_of(uint32_t word, int byte) {
  return __uint_as_float(byte == 3 ? word >> 1 : word << (23 - 8 * byte));
}

// Reduction over the two halves of a wave, in every lane.
template <typename F>
__device__ __forceinline__ float across_halves(float x, F f) {
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Reductions over the four quarters of a wave (the same row), in every lane.
template <typename F>
__device__ __forceinline__ float across_quarters(float x, F f) {
  // the swap of a register with itself leaves one half's values in both halves of either result
  u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Reduction over the 16 lanes of a quarter, in every lane.
template <typename F>
__device__ __forceinline__ int across_16(int x, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x128, 0xf, 0xf, false));   // rotations by 8, 4, 2, 1
  x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x124, 0xf, 0xf, false));
  x = f(x, __builtin_amdgcn_update_dpp(x, x, 0x122, 0xf, 0xf, false));
  return f(x, __builtin_amdgcn_update_dpp(x, x, 0x121, 0xf, 0xf, false));
}
// The same over the 32 lanes of a half.
template <typename F>
__device__ __forceinline__ int across_32(int x, F f) {
  x = across_16(x, f);
  const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false));
  return f((int)r[0], (int)r[1]);
}
__device__ __forceinline__ int min_of(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int max_of(int a, int b) { return a > b ? a : b; }

// Read through the scalar cache: the index is the same for the whole wave, and no launch writes what it reads here.
typedef const int32_t __attribute__((address_space(4)))* uniform_ints;
__device__ __forceinline__ uniform_ints uniform(const int32_t* p) { return (uniform_ints)(uintptr_t)p; }

// The context and the tile of `size` rows that a workgroup begins with, and how far down it goes on (AttendPlan).
struct Task {
  int seq, q0, q1, n_rows, tile, step;
  static __device__ __forceinline__ int within(const AttendArgs& a, int q) { return q < 0 ? 0 : q > a.total_q ? a.total_q : q; }
  __device__ __forceinline__ Task(const AttendArgs& a, int size) {
    const int slot = blockIdx.z * gridDim.y + blockIdx.y;
    seq = slot;
    int before = 0;                                  // tiles of the context whose places come first: the last rows see the most keys
    if (a.flat) {
      // contexts 1 .. n_seq - 1 that begin at this place or before it, by 64 lanes at once
      seq = 0;
      for (int left = a.n_seq - 1; left > 0;) {
        const int by = (left + 63) >> 6, s = seq + ((threadIdx.x & 63) + 1) * by;
        const bool begun = s < a.n_seq && within(a, a.cu_q[s]) * a.group / size + s <= slot;
        seq += __popcll(__ballot(begun)) * by;
        left = by > 1 ? by : 0;
      }
      seq = __builtin_amdgcn_readfirstlane(seq);
    }
    if (seq < a.n_seq) {
      q0 = within(a, uniform(a.cu_q)[seq]);
      q1 = within(a, uniform(a.cu_q)[seq + 1]);
      if (a.flat) before = slot - (q0 * a.group / size + seq);
    } else {
      seq = q0 = q1 = 0;
    }
    n_rows = (q1 - q0) * a.group;
    const int n_tiles = n_rows > 0 ? (n_rows + size - 1) / size : 0;
    tile = before < 0 ? -1 : n_tiles - 1 - before;
    step = a.flat ? 0x40000000 : 1;                  // more than there are tiles
  }
};

// Where runs of 16 keys of a KV head stand, 64 runs at a time: run i's offset is lane i's, worked out by all lanes at once (per
// run and wave the 64-bit products would be some 25 scalar instructions), and the entries of the 64 behind are on their
// way meanwhile.
struct Places {
  const int32_t* table;
  const uint8_t* pool;             // of the KV head
  int64_t num_pages;
  uint32_t page_bytes, sub_bytes;
  int max_blocks, block_shift;
  uint32_t lo, hi;
  uint64_t there;                  // runs whose page is one of the pool's
  int entry;

  __device__ __forceinline__ Places(const AttendArgs& a, int seq, int kvh, int sub)
      : table(a.block_tables + (size_t)seq * a.max_blocks), num_pages(a.num_pages), sub_bytes(sub), max_blocks(a.max_blocks), block_shift(a.block_shift) {
    const uint32_t head_bytes = (uint32_t)sub << (a.block_shift - 4);
    page_bytes = head_bytes * a.n_kv;
    pool = a.pool + (size_t)kvh * head_bytes;
  }
  // `key`: the lane's run's first key
  __device__ __forceinline__ void look_up(int key) {
    const int block = (int)((uint32_t)key >> block_shift);
    entry = table[block < max_blocks ? block : max_blocks - 1];
  }
  __device__ __forceinline__ void settle(int key) {
    const bool ok = entry >= 0 && entry < num_pages;
    there = __ballot(ok);
    const uint64_t at = (uint64_t)(uint32_t)(ok ? entry : 0) * page_bytes + ((key & ((1 << block_shift) - 1)) >> 4) * sub_bytes;
    lo = (uint32_t)at;
    hi = (uint32_t)(at >> 32);
  }
  __device__ __forceinline__ const uint8_t* of(int run) const {
    return pool + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, run) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, run));
  }
  // first byte of the run that `key` (the same for the wave) is in, null where there is no page (rare paths)
  __device__ __forceinline__ const uint8_t* run_of(int key) const {
    const int block = key >> block_shift, page = block < max_blocks ? table[block] : -1;
    if (page < 0 || page >= num_pages) return nullptr;
    return pool + (uint64_t)(uint32_t)page * page_bytes + ((key & ((1 << block_shift) - 1)) >> 4) * sub_bytes;
  }
};

// NaN if a row with keys lo .. hi sees, among keys [key0, key0 + n), one whose values are NaN in a group of 32 channels, else 0.
// All lanes go the same way: see the note on divergence in kv4_attend.hip.
template <int HD>
__device__ __forceinline__ float nan_values(const Places& places, int key0, int n, int lo, int hi, int group) {
  float poison = 0.f;
  for (int key = key0; key < key0 + n; ++key) {
    const uint8_t* at = places.run_of(key);
    if (!at) continue;
    const bool is = at[v_scales_at(HD) + ((key & 15) >> 2) * (HD / 8) + (key & 3) + 4 * group] == kNanScale && key >= lo && key <= hi;
    poison = is ? __builtin_nanf("") : poison;
  }
  return poison;
}

// A lane's bytes of 16 keys of a head.
template <int N>
__device__ __forceinline__ void load_words(uint32_t* to, const uint8_t* from) {
  if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(from);
    to[0] = x[0]; to[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(from + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) to[i + j] = x[j];
    }
  }
}
// K's scales as the word that they are in: of a byte the compiler would clear the other bits where the load is given its
// place in the loop, and wait for it there (64 contexts of up to 8192 keys: 81 us without, 88 with that wait).
template <int HD>
struct RawK {
  uint32_t w[HD / 32], scales;
  __device__ __forceinline__ void load(const uint8_t* at, int l16, int q4) {
    load_words<HD / 32>(w, at + (l16 * (HD / 2) + q4 * (HD / 8)));
    scales = *reinterpret_cast<const uint32_t*>(at + k_scales_at(HD) + ((l16 * (HD / 32) + q4 * HD / 128) & ~3));
  }
  // scale of word j; the lane's first byte of the word goes to the exponent's place in one turn
  __device__ __forceinline__ float scale(int l16, int q4, int j) const {
    const uint32_t first = ((l16 * (HD / 32) + q4 * HD / 128) & 3) * 8 + 9;
    return __uint_as_float(__builtin_rotateright32(scales, first + (HD == 256 ? 8 * (j >> 2) : 0)));
  }
};
template <int HD>
struct RawV {
  uint32_t w[HD / 32], scales;
  __device__ __forceinline__ void load(const uint8_t* at, int l16, int q4) {
    load_words<HD / 32>(w, at + (v_codes_at(HD) + (q4 * 16 + l16) * (HD / 8)));
    scales = *reinterpret_cast<const uint32_t*>(at + (v_scales_at(HD) + (q4 * (HD / 32) + l16 * HD / 512) * 4));
  }
};

// Values of 16 keys, a lane's four at `key`: those that no row sees (outside [begin, end), or without a page), and NaN, become zeros: weight 0
// times NaN would be NaN, whatever an unused place holds.  True if NaN was among those that a row may see.
template <int HD>
__device__ __forceinline__ bool only_seen(RawV<HD>& r, int key, int begin, int end, bool gone) {
  bool nan_value = false;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const bool none = gone || key + v < begin || key + v >= end, nan = (r.scales >> (8 * v) & 255u) == kNanScale;
    const uint32_t keep = none || nan ? 0u : 0xffffffffu;
    r.scales = (r.scales & ~(255u << (8 * v) & ~keep)) | (127u << (8 * v) & ~keep);
    if constexpr (HD == 64)       r.w[v >> 1] &= keep | (v & 1 ? 0x0000ffffu : 0xffff0000u);
    else if constexpr (HD == 128) r.w[v] &= keep;
    else { r.w[2 * v] &= keep; r.w[2 * v + 1] &= keep; }
    nan_value |= nan && !none;
  }
  return nan_value;
}

}  // namespace hc
