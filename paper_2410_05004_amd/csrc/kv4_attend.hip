// Attention over the 4-bit cache (layout: kv4.h).
//
// For a query row (token i of a context, head h) at position p, keys j in [lo, hi], lo = max(0, p - window + 1), hi = min(p, keys - 1):
//   w_j = exp(scale * q . k_j - top),   out = sum_j w_j v_j / sum_j w_j,   lse = top + log(sum_j w_j)
// in one pass over the keys with a running top and sum.  Everything is computed transposed: S^T = K Q^T and
// O^T = V^T W^T, so that a lane of a wave holds values of ONE row (column l16 of the matrix ops' results): the top and
// sum need no exchange between columns, and W goes from the result registers of the first product into the
// operand registers of the second as it stands -- key 4 * q4 + v of either half of 32 keys is register v of quarter q4
// there, and element v (+ 4) of its operand here, an order that V^T's operand has to share and the cache is laid out in.
// Decoded keys and values are exact in bf16; W is rounded to bf16 (2^-9 relative, without a bias, which averages out over
// the keys), sums and statistics are fp32.
#include "kv4.h"

namespace hc {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr float kNegInf = -__builtin_inff();
// The running top follows a row's maximum only when that has grown by more than this (of base 2): weights then reach
// 2^8 instead of 1, which costs nothing in floating point, and most steps rescale nothing.
constexpr float kTopSlack = 8.f;

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

__device__ __forceinline__ float across_quarters_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float across_quarters_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// A lane's bytes of 16 keys of a head.
template <int HD>
struct Raw {
  static constexpr int kWords = HD / 32;
  uint32_t k[kWords], v[kWords];
  uint32_t ks, vs;
};

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

// `at`: the 16 keys' first byte, the same for the whole wave
template <int HD>
__device__ __forceinline__ void load_raw(Raw<HD>& r, const uint8_t* at, int l16, int q4) {
  load_words<HD / 32>(r.k, at + l16 * (HD / 2) + q4 * (HD / 8));
  load_words<HD / 32>(r.v, at + v_codes_at(HD) + (q4 * 16 + l16) * (HD / 8));
  const uint8_t* ks = at + k_scales_at(HD) + l16 * (HD / 32);
  if constexpr (HD == 64)       r.ks = ks[q4 >> 1];
  else if constexpr (HD == 128) r.ks = ks[q4];
  else                          r.ks = *reinterpret_cast<const uint16_t*>(ks + 2 * q4);
  r.vs = *reinterpret_cast<const uint32_t*>(at + v_scales_at(HD) + (q4 * (HD / 32) + l16 * HD / 512) * 4);
}

// What the queries of 16 rows see.
struct Rows {
  int lo, hi;              // this lane's row: keys lo .. hi, none if hi < lo
  int begin, end;          // of all rows: keys that any row sees
  int all_lo, all_hi;      // keys that every row sees
};

// Steps of 32 keys [step, ...) of one wave, every `stride`-th, for 16 rows.
template <int HD>
struct Walk {
  const AttendArgs& a;
  const int32_t* table;
  const uint8_t* pool;           // of the KV head
  int64_t page_bytes;
  int keys;                      // of the context
  int bad = 0;

  // first byte of keys [key, key + 16), and 0 in `ok` where the page is none of the pool's
  __device__ __forceinline__ const uint8_t* place(int key, bool& ok) {
    const int block = key >> a.block_shift;
    int page = block < a.max_blocks ? table[block] : 0;
    ok = page >= 0 && page < a.num_pages;
    if (!ok) page = 0;
    return pool + page * page_bytes + ((key & ((1 << a.block_shift) - 1)) >> 4) * sub_bytes(HD);
  }
};

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) { const int o = __shfl_xor(x, m); x = x < o ? x : o; }
  return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) { const int o = __shfl_xor(x, m); x = x > o ? x : o; }
  return x;
}

// Rows of a context and KV head: row r is query r / group, query head r % group of the KV head's.  A workgroup takes 16
// rows and a share of the keys, its four waves every fourth step of 32 keys.
template <int HD>
__global__ __launch_bounds__(256) void attend_few_kernel(const AttendArgs a) {
  constexpr int kSteps = HD / 32;         // matrix ops along the channels
  constexpr int kSlices = HD / 16;        // blocks of 16 channels of the result
  __shared__ float s_out[3][kSlices * 4][64];
  __shared__ float s_top[4][16], s_sum[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q4 = lane >> 4;
  const int split = blockIdx.x % a.n_split, kvh = blockIdx.x / a.n_split, seq = blockIdx.z;
  int q0 = a.cu_q[seq], q1 = a.cu_q[seq + 1];
  q0 = q0 < 0 ? 0 : q0;
  q1 = q1 > a.total_q ? a.total_q : q1;
  const int64_t most = (int64_t)a.max_blocks << a.block_shift;
  int keys = a.kv_lens[seq];
  if (keys > most || keys < 0) {
    if (threadIdx.x == 0) atomicOr(a.err, HC_DEV_BAD_POSITION);
    keys = keys < 0 ? 0 : (int)most;
  }
  const int n_rows = (q1 - q0) * a.group;
  const int32_t* table = a.block_tables + (size_t)seq * a.max_blocks;
  const int subs = 1 << (a.block_shift - 4);
  const int64_t head_bytes = (int64_t)subs * sub_bytes(HD);
  Walk<HD> walk{a, table, a.pool + kvh * head_bytes, head_bytes * a.n_kv, keys};

  for (int tile = blockIdx.y; tile * 16 < n_rows; tile += gridDim.y) {
    // ---- the rows
    const int r = tile * 16 + l16;
    const bool row_in = r < n_rows;
    const int rr = row_in ? r : n_rows - 1;
    const int qi = rr / a.group, head = kvh * a.group + rr - qi * a.group;
    const int64_t tok = q0 + qi;
    const int pos = a.positions[tok];
    Rows rows;
    rows.hi = pos < keys - 1 ? pos : keys - 1;
    rows.lo = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
    const bool sees = rows.hi >= rows.lo;
    rows.begin = wave_min(sees ? rows.lo : 0x7fffffff);
    rows.end = wave_max(sees ? rows.hi + 1 : 0);
    rows.all_lo = wave_max(rows.lo);
    rows.all_hi = wave_min(rows.hi);
    bf16x8 q[kSteps];
    {
      const uint16_t* from = a.q + tok * a.q_stride + head * HD + q4 * (HD / 4);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) q[j] = *reinterpret_cast<const bf16x8*>(from + 8 * j);
    }
    // ---- this workgroup's share of the keys, in steps of 32
    const int first = rows.begin < rows.end ? rows.begin >> 5 : 0;
    const int n_step = rows.begin < rows.end ? ((rows.end + 31) >> 5) - first : 0;
    const int share = (n_step + a.n_split - 1) / a.n_split;
    int step = first + split * share;
    int stop = step + share;
    if (stop > first + n_step) stop = first + n_step;
    step += wave;

    f32x4 o[kSlices];
#pragma unroll
    for (int b = 0; b < kSlices; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = kNegInf, top_used = 0.f, sum = 0.f;     // top_used: 0 while there is no finite top, so that exp2 of -inf stays 0

    Raw<HD> raw[2], next[2];
    bool ok[2], next_ok[2];
    if (step < stop) {
#pragma unroll
      for (int h = 0; h < 2; ++h) load_raw<HD>(raw[h], walk.place(step * 32 + 16 * h, ok[h]), l16, q4);
    }
    for (; step < stop; step += 4) {
      if (step + 4 < stop) {
#pragma unroll
        for (int h = 0; h < 2; ++h) load_raw<HD>(next[h], walk.place((step + 4) * 32 + 16 * h, next_ok[h]), l16, q4);
      }
      const int key0 = step * 32;
      // ---- S^T = K Q^T
      f32x4 s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const float ks = scale_of(raw[h].ks, HD == 256 ? j >> 2 : 0);
          u32x4 k;
#pragma unroll
          for (int i = 0; i < 4; ++i) k[i] = decode2(raw[h].k[j], ks, i);
          s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), q[j], s[h], 0, 0, 0);
        }
      }
      // ---- masks, where a row's first or last key lies in these 32 or a page is missing
      if (key0 < rows.all_lo || key0 + 31 > rows.all_hi || !ok[0] || !ok[1]) {
        bool nan_value = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!ok[h] && key0 + 16 * h < rows.end && key0 + 16 * h + 15 >= rows.begin) walk.bad = HC_DEV_BAD_PAGE;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int key = key0 + 16 * h + 4 * q4 + v;
            if (!ok[h] || key < rows.lo || key > rows.hi) s[h][v] = kNegInf;
            // V of a key that no row sees is taken as zero, whatever its place holds: weight 0 times NaN would be NaN
            const bool none = !ok[h] || key < rows.begin || key >= rows.end;
            const uint32_t byte = raw[h].vs >> (8 * v) & 255u;
            if (none || byte == kNanScale) {
              raw[h].vs = (raw[h].vs & ~(255u << (8 * v))) | 127u << (8 * v);
              if constexpr (HD == 64)       raw[h].v[v >> 1] &= v & 1 ? 0x0000ffffu : 0xffff0000u;
              else if constexpr (HD == 128) raw[h].v[v] = 0;
              else                          raw[h].v[2 * v] = raw[h].v[2 * v + 1] = 0;
              nan_value |= !none;
            }
          }
        }
        // NaN among the values of keys that some row sees: taken out above, and given to the rows that see them here
        if (__any(nan_value)) {
          for (int h = 0; h < 2; ++h) {
            bool ok_h;
            const uint8_t* at = walk.place(key0 + 16 * h, ok_h) + v_scales_at(HD);
            if (!ok_h) continue;
            for (int t = 0; t < 16; ++t) {
              const int key = key0 + 16 * h + t;
              if (key < rows.lo || key > rows.hi) continue;
              // this lane's results are channels q4 * HD / 4 ..
#pragma unroll
              for (int g = 0; g < (HD == 256 ? 2 : 1); ++g) {
                const int group = HD == 64 ? q4 >> 1 : HD == 128 ? q4 : 2 * q4 + g;
                if (at[((t >> 2) * (HD / 32) + group) * 4 + (t & 3)] != kNanScale) continue;
#pragma unroll
                for (int b = 0; b < kSlices; ++b)
#pragma unroll
                  for (int v = 0; v < 4; ++v)
                    if (HD != 256 || (v >> 1) == g) o[b][v] = __builtin_nanf("");
              }
            }
          }
        }
      }
      // ---- running top and sum
      float m = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      m *= a.scale_log2;
      if (__any(m > top + kTopSlack)) {
        const float grown = fmaxf(top, across_quarters_max(m));
        const float used = grown == kNegInf ? 0.f : grown;
        const float shrink = __builtin_amdgcn_exp2f(top - used);        // 0 for the first keys
        top = grown;
        top_used = used;
        sum *= shrink;
#pragma unroll
        for (int b = 0; b < kSlices; ++b) o[b] *= shrink;
      }
      bf16x8 w;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][v], a.scale_log2, -top_used));
          sum += e;
          w[4 * h + v] = (__bf16)e;
        }
      // ---- O^T += V^T W^T: byte i of a key's word holds slices 2 i and 2 i + 1
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        u32x4 even, odd;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t c[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int byte = t * (HD / 32) + i;
            c[t] = decode2(raw[h].v[byte >> 2], scale_of(raw[h].vs, t), byte & 3);
          }
          even[2 * h] = __builtin_amdgcn_perm(c[1], c[0], 0x05040100);
          even[2 * h + 1] = __builtin_amdgcn_perm(c[3], c[2], 0x05040100);
          odd[2 * h] = __builtin_amdgcn_perm(c[1], c[0], 0x07060302);
          odd[2 * h + 1] = __builtin_amdgcn_perm(c[3], c[2], 0x07060302);
        }
        o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), w, o[2 * i], 0, 0, 0);
        o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), w, o[2 * i + 1], 0, 0, 0);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) { raw[h] = next[h]; ok[h] = next_ok[h]; }
    }
    if (walk.bad && lane == 0) atomicOr(a.err, walk.bad);

    // ---- the four waves' shares, added up in the waves' order
    sum = across_quarters_sum(sum);
    if (q4 == 0) { s_top[wave][l16] = top; s_sum[wave][l16] = sum; }
    __syncthreads();
    float best = kNegInf;
#pragma unroll
    for (int i = 0; i < 4; ++i) best = fmaxf(best, s_top[i][l16]);
    const float best_used = best == kNegInf ? 0.f : best;
    const float mine = __builtin_amdgcn_exp2f(top - best_used);
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) total += s_sum[i][l16] * __builtin_amdgcn_exp2f(s_top[i][l16] - best_used);
    if (wave > 0) {
#pragma unroll
      for (int b = 0; b < kSlices; ++b)
#pragma unroll
        for (int v = 0; v < 4; ++v) s_out[wave - 1][b * 4 + v][lane] = o[b][v] * mine;
    }
    __syncthreads();
    if (wave == 0 && row_in) {
      const int64_t row = tok * a.n_q + head;
      // register (b, v) is channel (4 * q4 + v) * HD / 16 + b
      if (a.n_split == 1) {
        const float norm = total == 0.f ? 0.f : 1.f / total;         // a row that sees no key: zeros
        uint16_t* to = a.out + tok * a.out_stride + head * HD + q4 * (HD / 4);
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int b = 0; b < kSlices; b += 4) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[i] = (((o[b + i][v] * mine + s_out[0][(b + i) * 4 + v][lane]) + s_out[1][(b + i) * 4 + v][lane]) + s_out[2][(b + i) * 4 + v][lane]) * norm;
            u32x2 y;
            y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[0], x[1]}, bf16x2));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2], x[3]}, bf16x2));
            *reinterpret_cast<u32x2*>(to + v * kSlices + b) = y;
          }
        if (a.lse && q4 == 0) a.lse[row] = best_used * 0.69314718056f + __logf(total);
      } else {
        const int64_t n_row = (int64_t)a.total_q * a.n_q;
        float* to = a.part + (split * n_row + row) * HD + q4 * (HD / 4);
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int b = 0; b < kSlices; b += 4) {
            f32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              x[i] = ((o[b + i][v] * mine + s_out[0][(b + i) * 4 + v][lane]) + s_out[1][(b + i) * 4 + v][lane]) + s_out[2][(b + i) * 4 + v][lane];
            *reinterpret_cast<f32x4*>(to + v * kSlices + b) = x;
          }
        if (q4 == 0) {
          float* ml = a.part + a.n_split * n_row * HD + (split * n_row + row) * 2;
          ml[0] = best;
          ml[1] = total;
        }
      }
    }
    __syncthreads();
  }
}

// Joins the shares of a row, in their order: a wave a row.
template <int HD>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t n_row = (int64_t)a.total_q * a.n_q;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= n_row) return;
  const int64_t tok = row / a.n_q;
  const int head = (int)(row - tok * a.n_q);
  if (tok < a.cu_q[0] || tok >= a.cu_q[a.n_seq]) return;    // no context's
  const float* ml = a.part + a.n_split * n_row * HD + row * 2;
  float best = kNegInf;
  for (int i = lane; i < a.n_split; i += 64) best = fmaxf(best, ml[i * n_row * 2]);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) best = fmaxf(best, __shfl_xor(best, m));
  const float used = best == kNegInf ? 0.f : best;
  float total = 0.f;
  constexpr int kPer = HD / 64;
  float x[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = 0.f;
  for (int i = 0; i < a.n_split; ++i) {
    const float w = __builtin_amdgcn_exp2f(ml[i * n_row * 2] - used);
    total += w * ml[i * n_row * 2 + 1];
    const float* from = a.part + (i * n_row + row) * HD + lane * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] += w * from[e];
  }
  const float norm = total == 0.f ? 0.f : 1.f / total;
  uint16_t* to = a.out + tok * a.out_stride + head * HD + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) to[e] = __builtin_bit_cast(uint16_t, (__bf16)(x[e] * norm));
  if (a.lse && lane == 0) a.lse[row] = used * 0.69314718056f + __logf(total);
}

bool attend_head_dim(int head_dim) { return head_dim == 64 || head_dim == 128 || head_dim == 256; }

AttendPlan plan_attend(int n_q, int n_kv, int head_dim, int n_seq, int total_q, int max_q, int max_kv) {
  AttendPlan p;
  const int group = n_q / n_kv;
  int64_t tiles = ((int64_t)max_q * group + 15) / 16;
  p.row_tiles = (int)(tiles < 1 ? 1 : tiles > 65535 ? 65535 : tiles);
  const int64_t base = (int64_t)n_seq * n_kv * p.row_tiles;
  // keys are split until there are some 4096 workgroups, not below 256 keys to one
  int64_t split = base > 0 ? 4096 / base : 1, most = ((int64_t)max_kv + 255) / 256;
  if (split > most) split = most;
  if (split > 512) split = 512;
  p.n_split = split < 1 ? 1 : (int)split;
  p.workspace = p.n_split > 1 ? (int64_t)p.n_split * total_q * n_q * (head_dim + 2) * 4 : 0;
  return p;
}

template <int HD>
static void launch_hd(const AttendArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(attend_few_kernel<HD>, dim3(a.n_split * a.n_kv, a.row_tiles, a.n_seq), dim3(256), 0, stream, a);
  if (a.n_split > 1) {
    const int64_t n_row = (int64_t)a.total_q * a.n_q;
    hipLaunchKernelGGL(attend_join_kernel<HD>, dim3((unsigned)((n_row + 3) / 4)), dim3(256), 0, stream, a);
  }
}

hipError_t launch_attend(const AttendArgs& a, int head_dim, hipStream_t stream) {
  if (a.total_q <= 0 || a.n_seq <= 0) return hipSuccess;
  switch (head_dim) {
    case 64: launch_hd<64>(a, stream); break;
    case 128: launch_hd<128>(a, stream); break;
    case 256: launch_hd<256>(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hc
