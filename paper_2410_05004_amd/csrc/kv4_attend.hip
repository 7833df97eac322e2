// Attention over the 4-bit cache (layout: kv4.h).
//
// For a query row (token i of a context, head h) at position p, keys j in [lo, hi], lo = max(0, p - window + 1), hi = min(p, keys - 1):
//   w_j = exp(scale * q . k_j - top),   out = sum_j w_j v_j / sum_j w_j,   lse = top + log(sum_j w_j)
// in one pass over the keys with a running top and sum.  Everything is computed transposed: S^T = K Q^T and
// O^T = V^T W^T, so that a lane of a wave holds values of ONE row (column l16 of the matrix ops' results): the top and
// sum need no exchange between columns, and W goes from the result registers of the first product into the
// operand registers of the second as it stands -- key 4 * q4 + v of either half of 32 keys is register v of quarter q4
// there, and element v (+ 4) of its operand here, an order that V^T's operand has to share and the cache is laid out in.
// No lane of a wave goes another way than the others while results are in registers: where these are many, the compiler
// has been seen to put a copy that it needs for all lanes into a branch that some had not taken (sums of the second 16 rows were
// wrong at 256 channels, the registers in question traced in the generated code).  What concerns some lanes is selected, and what
// several would store alike they all do.
// Decoded keys and values are exact in bf16; W is rounded to bf16 (2^-8 relative at most, without a bias, which averages out over
// the keys), in two parts where rows are few (see PAIRED); sums and statistics are fp32.
#include <algorithm>
#include <climits>

#include "kv4_device.h"

namespace hc {

// Rows of a context and KV head: row r is query r / group, query head r % group of the KV head's.  A workgroup takes
// NB blocks of 16 rows and a share of the keys; its waves take every so-many-th step of 32 keys, for all the rows.
// The next step's bytes are fetched into the registers as soon as this step's are decoded: keys before the softmax, values
// behind the second product.
// Bound, single tokens: memory, where there are keys enough (32 heads over 8 of 128: 64 contexts of up to 8192 keys, 374 MB, 82 us, 4.6 TB/s; 64
// heads over 8, one context of 131072 keys, 143 MB, 26.5 us, 5.4 TB/s; a large sum reads 5.6); else latency: one context of 1037 keys 11.1 us,
// of which 5.8 for the launch, the lengths, the table and the first keys, and 0.5 to 0.6 for each step of the four waves.  Some 16 rows: 4 waves
// are better than 8 or 16 (64 contexts of up to 4000 keys 38, 41, 58 us; one of 1000 9.9, 9.9, 15).
//
// Weights are rounded to bf16 for the second product.  Where a call's contexts have up to 8 rows, half of a block's 16 columns would compute
// a row twice: PAIRED, columns 8 .. 15 take the same rows with what the rounding took from the weights, to bf16 again, and the two halves
// are added at the end: 2^-17 at most is lost then (in norm outputs are off by 0.0017 as if rounded once, instead of 0.0023).  Costs 2.5
// instructions a weight: one context of 1037 keys 10.8 us without, 11.1 with, the 64 contexts 80.4 and 82.4.  A second product over the same
// columns costs more (11.6 and 84.6; one context's 1024 queries on 4000 keys 95 us instead of 75), so other calls have the rounded weights alone.
constexpr int kFewWaves = 4;
template <int HD, int NB, bool PAIRED>
__global__ __launch_bounds__(64 * kFewWaves, NB * HD <= 128 ? 3 : NB * HD <= 256 ? 2 : 1) void attend_kernel(const AttendArgs a) {
  constexpr int kSteps = HD / 32;         // matrix ops along the channels
  constexpr int kSlices = HD / 16;        // blocks of 16 channels of the result
  __shared__ float s_out[kFewWaves / 2][kSlices * 4][64];
  __shared__ float s_top[kFewWaves][NB][16], s_sum[kFewWaves][NB][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, q4 = lane >> 4;
  const int split = blockIdx.x % a.n_split, kvh = blockIdx.x / a.n_split;
  const Task task(a, NB * 16);
  const int seq = task.seq, q0 = task.q0, n_rows = task.n_rows;
  const bool paired = PAIRED && n_rows <= kPairedRows;
  // of a pair of rounded weights, what a lane's column takes from the weights themselves: the first or second, or nothing
  const bool rest = paired && l16 >= kPairedRows;
  const uint32_t first_of = rest ? 0x01000c0cu : 0x0c0c0c0cu, second_of = rest ? 0x03020c0cu : 0x0c0c0c0cu;
  const int64_t room = (int64_t)a.max_blocks << a.block_shift, most = room < kMaxKeys ? room : kMaxKeys;
  int keys = uniform(a.kv_lens)[seq];
  if (keys > most || keys < 0) {
    if (threadIdx.x == 0) atomicOr(a.err, HC_DEV_BAD_POSITION);
    keys = keys < 0 ? 0 : (int)most;
  }
  if (task.tile < 0) return;                         // not before the count is asked for: both are on their way together
  Places places(a, seq, kvh, sub_bytes(HD));
  bool bad_page = false;

  for (int tile = task.tile; tile >= 0; tile -= task.step) {
    // ---- this workgroup's share of the keys, in steps of 32: of all that there are, or, if there is a window, of those that any row
    // sees.  Without one nothing waits for the positions: the table's entries and the rows are on their way together.
    auto query_of = [&](int nb) __attribute__((always_inline)) {
      const int r = (tile * NB + nb) * 16 + (paired ? l16 & 7 : l16);
      return (r < n_rows ? r : n_rows - 1) / a.group;
    };
    auto head_of = [&](int nb, int query) __attribute__((always_inline)) {
      const int r = (tile * NB + nb) * 16 + (paired ? l16 & 7 : l16);
      return kvh * a.group + (r < n_rows ? r : n_rows - 1) - query * a.group;
    };
    const int lane_key = (lane >> 1) * 32 * kFewWaves + (lane & 1) * 16;        // run i of a round: half i % 2 of this wave's step i / 2
    int first = 0, n_step = (keys + 31) >> 5, share = 0, step = 0, stop = 0;
    auto take_share = [&]() __attribute__((always_inline)) {
      share = (n_step + a.n_split - 1) / a.n_split;
      step = first + split * share;
      stop = min_of(step + share, first + n_step);
      step += wave;
      if (step < stop) places.look_up(step * 32 + lane_key);
    };
    if (a.window == 0) take_share();
    // ---- the rows
    int lo[NB], hi[NB];                              // keys that this lane's rows see: none if hi < lo
    int begin = 0x7fffffff, end = 0, all_lo = 0, all_hi = 0x7fffffff;   // keys that any row sees, and that every row sees
    bf16x8 q[NB][kSteps];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int qi = query_of(nb), pos = a.positions[q0 + qi];
      const uint16_t* from = a.q + (q0 + qi) * a.q_stride + head_of(nb, qi) * HD + q4 * (HD / 4);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) q[nb][j] = *reinterpret_cast<const bf16x8*>(from + 8 * j);
      hi[nb] = pos < keys - 1 ? pos : keys - 1;
      lo[nb] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
      const bool sees = hi[nb] >= lo[nb];
      begin = min_of(begin, sees ? lo[nb] : 0x7fffffff);
      end = max_of(end, sees ? hi[nb] + 1 : 0);
      all_lo = max_of(all_lo, lo[nb]);
      all_hi = min_of(all_hi, hi[nb]);
    }
    begin = __builtin_amdgcn_readfirstlane(across_16(begin, min_of));
    end = __builtin_amdgcn_readfirstlane(across_16(end, max_of));
    all_lo = __builtin_amdgcn_readfirstlane(across_16(all_lo, max_of));
    all_hi = __builtin_amdgcn_readfirstlane(across_16(all_hi, min_of));
    if (a.window != 0) {
      first = begin < end ? begin >> 5 : 0;
      n_step = begin < end ? ((end + 31) >> 5) - first : 0;
      take_share();
    }
    stop = min_of(stop, (end + 31) >> 5);

    f32x4 o[NB][kSlices];
    float top[NB], used[NB], sum[NB];                // used: the top, 0 while there is no finite one, so that exp2 of -inf stays 0
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      top[nb] = kNegInf;
      used[nb] = sum[nb] = 0.f;
#pragma unroll
      for (int b = 0; b < kSlices; ++b) o[nb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    RawK<HD> rk[2];
    RawV<HD> rv[2];
    int at = 0, gone = 0, next_gone = 0;             // run of the next fetch; halves without a page, of this step and the next
    auto next_runs = [&](int s) __attribute__((always_inline)) {       // places of step s
      if (at == 0) {
        places.settle(s * 32 + lane_key);
        places.look_up((s + 32 * kFewWaves) * 32 + lane_key);
      }
      next_gone = ~(int)(places.there >> at) & 3;
    };
    if (step < stop) {
      next_runs(step);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        rk[h].load(places.of(h), l16, q4);
        rv[h].load(places.of(h), l16, q4);
      }
      at = 2;
    }
    for (; step < stop; step += kFewWaves) {
      const int key0 = step * 32;
      gone = next_gone;
      next_runs(step + kFewWaves);                           // behind the last step: some page's, not used
      const uint8_t* next_at[2] = {places.of(at), places.of(at + 1)};
      at = (at + 2) & 63;
      // ---- S^T = K Q^T
      f32x4 s[NB][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          const float ks = rk[h].scale(l16, q4, j);
          u32x4 k;
#pragma unroll
          for (int i = 0; i < 4; ++i) k[i] = decode2(rk[h].w[j], ks, i);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            s[nb][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), q[nb][j], s[nb][h], 0, 0, 0);
          }
        }
        rk[h].load(next_at[h], l16, q4);
      }
      // ---- masks, where a row's first or last key lies in these 32 or a page is missing
      if (key0 < all_lo || key0 + 31 > all_hi || gone) {
        asm volatile("");                            // stays a branch: the compiler would mask every step
        bool nan_value = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool none = gone >> h & 1;
          if (none && key0 + 16 * h < end && key0 + 16 * h + 15 >= begin) bad_page = true;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int key = key0 + 16 * h + 4 * q4 + v;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              if (none || key < lo[nb] || key > hi[nb]) s[nb][h][v] = kNegInf;
          }
          nan_value |= only_seen<HD>(rv[h], key0 + 16 * h + 4 * q4, begin, end, none);
        }
        if (__any(nan_value)) {                      // taken out above, given to the rows that see it here
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            // this lane's results are channels q4 * HD / 4 ..: one group of 32, or two
            f32x2 poison;
#pragma unroll
            for (int g = 0; g < 2; ++g) poison[g] = nan_values<HD>(places, key0, 32, lo[nb], hi[nb], HD == 256 ? 2 * q4 + g : q4 * HD / 128);
#pragma unroll
            for (int b = 0; b < kSlices; ++b)
#pragma unroll
              for (int v = 0; v < 4; ++v) o[nb][b][v] += poison[v >> 1];
          }
        }
      }
      // ---- running top and sum
      bf16x8 w[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const f32x4 x = s[nb][0], y = s[nb][1];
        float m = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])));
        m *= a.scale_log2;
        if (__any(m > top[nb] + kTopSlack)) {
          const float grown = fmaxf(top[nb], across_quarters(m, [](float p, float r) { return fmaxf(p, r); }));
          used[nb] = grown == kNegInf ? 0.f : grown;
          const float shrink = __builtin_amdgcn_exp2f(top[nb] - used[nb]);        // 0 for the first keys
          top[nb] = grown;
          sum[nb] *= shrink;
#pragma unroll
          for (int b = 0; b < kSlices; ++b) o[nb][b] *= shrink;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int v = 0; v < 4; v += 2) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][h][v], a.scale_log2, -used[nb]));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nb][h][v + 1], a.scale_log2, -used[nb]));
            sum[nb] += e0;
            sum[nb] += e1;
            bf16x2 p = __builtin_convertvector(f32x2{e0, e1}, bf16x2);
            if constexpr (PAIRED) {
              const uint32_t bits = __builtin_bit_cast(uint32_t, p);
              p = __builtin_convertvector(f32x2{e0 - __uint_as_float(__builtin_amdgcn_perm(0, bits, first_of)),
                                                e1 - __uint_as_float(__builtin_amdgcn_perm(0, bits, second_of))}, bf16x2);
            }
            w[nb][4 * h + v] = p[0];
            w[nb][4 * h + v + 1] = p[1];
          }
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
            c[t] = decode2(rv[h].w[byte >> 2], scale_of(rv[h].scales, t), byte & 3);
          }
          even[2 * h] = __builtin_amdgcn_perm(c[1], c[0], 0x05040100);
          even[2 * h + 1] = __builtin_amdgcn_perm(c[3], c[2], 0x05040100);
          odd[2 * h] = __builtin_amdgcn_perm(c[1], c[0], 0x07060302);
          odd[2 * h + 1] = __builtin_amdgcn_perm(c[3], c[2], 0x07060302);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          o[nb][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), w[nb], o[nb][2 * i], 0, 0, 0);
          o[nb][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), w[nb], o[nb][2 * i + 1], 0, 0, 0);
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) rv[h].load(next_at[h], l16, q4);
    }

    // ---- the waves' shares, added up by halves: an order that is always the same
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      sum[nb] = across_quarters(sum[nb], [](float p, float r) { return p + r; });
      s_top[wave][nb][l16] = top[nb];                // from all four quarters
      s_sum[wave][nb][l16] = sum[nb];
    }
    __syncthreads();
    float best[NB], total[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      best[nb] = kNegInf;
      total[nb] = 0.f;
#pragma unroll
      for (int i = 0; i < kFewWaves; ++i) best[nb] = fmaxf(best[nb], s_top[i][nb][l16]);
      const float best_used = best[nb] == kNegInf ? 0.f : best[nb];
#pragma unroll
      for (int i = 0; i < kFewWaves; ++i) total[nb] += s_sum[i][nb][l16] * __builtin_amdgcn_exp2f(s_top[i][nb][l16] - best_used);
      const float mine = __builtin_amdgcn_exp2f(top[nb] - best_used);
#pragma unroll
      for (int b = 0; b < kSlices; ++b) o[nb][b] *= mine;
#pragma unroll
      for (int n = kFewWaves / 2; n > 0; n >>= 1) {
        if (wave >= n && wave < 2 * n) {
#pragma unroll
          for (int b = 0; b < kSlices; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) s_out[wave - n][b * 4 + v][lane] = o[nb][b][v];
        }
        __syncthreads();
        if (wave < n) {
#pragma unroll
          for (int b = 0; b < kSlices; ++b)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[nb][b][v] += s_out[wave][b * 4 + v][lane];
        }
        __syncthreads();
      }
    }
    if (wave == 0) {
      if (paired) {
#pragma unroll
        for (int b = 0; b < kSlices; ++b)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            o[0][b][v] += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(o[0][b][v]), 0x128, 0xf, 0xf, false));
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if ((tile * NB + nb) * 16 >= n_rows) continue;       // places behind the last row have computed that row too and store the same
        const int qi = query_of(nb), head = head_of(nb, qi);
        const int64_t tok = q0 + qi, row = tok * a.n_q + head;
        // register (b, v) is channel (4 * q4 + v) * HD / 16 + b
        if (a.n_split == 1) {
          const float norm = total[nb] == 0.f ? 0.f : 1.f / total[nb];         // a row that sees no key: zeros
          uint16_t* to = a.out + tok * a.out_stride + head * HD + q4 * (HD / 4);
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int b = 0; b < kSlices; b += 4) {
              u32x2 y;
              y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[nb][b][v] * norm, o[nb][b + 1][v] * norm}, bf16x2));
              y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[nb][b + 2][v] * norm, o[nb][b + 3][v] * norm}, bf16x2));
              *reinterpret_cast<u32x2*>(to + v * kSlices + b) = y;
            }
          if (a.lse) a.lse[row] = (best[nb] == kNegInf ? 0.f : best[nb]) * 0.69314718056f + __logf(total[nb]);
        } else {
          const int64_t n_row = (int64_t)a.total_q * a.n_q;
          float* to = a.part + (split * n_row + row) * HD + q4 * (HD / 4);
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int b = 0; b < kSlices; b += 4)
              *reinterpret_cast<f32x4*>(to + v * kSlices + b) = f32x4{o[nb][b][v], o[nb][b + 1][v], o[nb][b + 2][v], o[nb][b + 3][v]};
          *reinterpret_cast<f32x2*>(a.part + a.n_split * n_row * HD + (split * n_row + row) * 2) = f32x2{best[nb], total[nb]};
        }
      }
    }
    __syncthreads();
  }
  if (bad_page && lane == 0) atomicOr(a.err, HC_DEV_BAD_PAGE);
}

// Joins the shares of a row, in an order that depends on the sizes alone.  16 lanes read a share, HD / 16 channels each; PARTS such
// groups go over a row's shares, every PARTS-th, and 16 / PARTS rows are a workgroup's.  Bound: latency for few rows (64 rows of 64 shares 4 us),
// else the reads of the shares (64128 rows of 4: 9.7 us, 3.5 TB/s, out of the caches for the most part).
template <int HD, int PARTS>
__global__ __launch_bounds__(256) void attend_join_kernel(const AttendArgs a) {
  constexpr int kPer = HD / 16, kRows = 16 / PARTS;
  __shared__ float s_x[16][HD + 4], s_total[16];
  const int group = threadIdx.x >> 4, part = group % PARTS, l16 = threadIdx.x & 15;
  const int64_t n_row = (int64_t)a.total_q * a.n_q;
  int64_t row = (int64_t)blockIdx.x * kRows + group / PARTS;
  const bool in = row < n_row;
  row = in ? row : n_row - 1;
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part + a.n_split * n_row * HD) + row;
  float best = kNegInf;
  for (int i = l16; i < a.n_split; i += 16) best = fmaxf(best, ml[i * n_row][0]);
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) best = fmaxf(best, __shfl_xor(best, m));
  const float used = best == kNegInf ? 0.f : best;
  float total = 0.f;
  f32x4 x[kPer / 4];
#pragma unroll
  for (int e = 0; e < kPer / 4; ++e) x[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int i = part; i < a.n_split; i += PARTS) {
    const f32x2 t = ml[i * n_row];
    const float w = __builtin_amdgcn_exp2f(t[0] - used);
    total += w * t[1];
    const f32x4* from = reinterpret_cast<const f32x4*>(a.part + (i * n_row + row) * HD + l16 * kPer);
#pragma unroll
    for (int e = 0; e < kPer / 4; ++e) x[e] += w * from[e];
  }
#pragma unroll
  for (int e = 0; e < kPer / 4; ++e) *reinterpret_cast<f32x4*>(&s_x[group][l16 * kPer + 4 * e]) = x[e];
  if (l16 == 0) s_total[group] = total;
  __syncthreads();
  // the row's lanes take its channels
  const int first = group / PARTS * PARTS;
  const int64_t tok = row / a.n_q;
  const int head = (int)(row - tok * a.n_q);
  if (!in || tok < uniform(a.cu_q)[0] || tok >= uniform(a.cu_q)[a.n_seq]) return;    // no context's
  total = 0.f;
#pragma unroll
  for (int i = 0; i < PARTS; ++i) total += s_total[first + i];
  const float norm = total == 0.f ? 0.f : 1.f / total;
  const int lane = threadIdx.x - first * 16;
  for (int c = lane; c < HD; c += PARTS * 16) {
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) y += s_x[first + i][c];
    a.out[tok * a.out_stride + head * HD + c] = __builtin_bit_cast(uint16_t, (__bf16)(y * norm));
  }
  if (a.lse && lane == 0) a.lse[row] = used * 0.69314718056f + __logf(total);
}

bool attend_head_dim(int head_dim) { return head_dim == 64 || head_dim == 128 || head_dim == 256; }

// Blocks of 16 rows of a workgroup, for `blocks` of them in all contexts and KV heads and `tiles` of kv4_prompt.hip's workgroups.
// `some`: contexts have more than one block; `filled`: they fill those tiles.
// Measured, 32 heads of 128 over 8 KV heads unless said otherwise, microseconds with 1 | 2 blocks | that kernel:
// - one context, 16 queries, 1000 keys 10.2 | 12.8, 64 queries, 1000 keys 10.2 | 12.9, 256 queries, 1000 keys 13.2 | 13.3; 64 queries,
//   8000 keys 27.8 | 25.6; 1024 queries, 16000 keys 392 | 307; 14 heads of 64 over 2, 64 queries, 8000 keys 15.1 | 15.0, 1024 queries,
//   4000 keys 41 | 32: keys are decoded once for 32 rows, and half as many waves wait for memory at once, so 2 blocks from some
//   800 000 pairs of a block and a key on (64 contexts of 4 queries, 2000 keys 23 | 27: not for 16 rows).  256 channels take registers
//   for one wave of a SIMD then: 16 heads over 8, 64 queries, 8000 keys 31 | 48, 8 contexts of 1024, 2048 keys 296 | 448 | 322: always 1.
// - kv4_prompt.hip decodes for 128 or 256 rows, but starts late (30 us with next to no keys) and has two workgroups on a compute unit:
//   8 contexts of 256 queries, 1000 keys 50 | 49 | 38; of 64 queries, 4000 keys 45 | 39 | 50; of 1024 queries, 2048 keys 298 | 247 | 205;
//   64 of 128 queries, 4000 keys 576 | 469 | 397; one of 1024, 1024 keys 27 | 26 | 33, 4000 keys 100 | 77 | 87, 16000 keys
//   392 | 307 | 277; one of 256, 16000 keys 118 | 102 | 93; 64 of 16 (64 rows) 55 | 48 | 65: if its tiles are filled to three quarters,
//   and there are two for every compute unit, or fewer than one and keys enough for shares of 1024 at least.
static int row_blocks(int head_dim, int64_t blocks, int64_t keys, int64_t tiles, bool some, bool filled) {
  const bool wide = head_dim == 256;
  if (!wide && filled && (tiles >= 2 * kChipCUs || (tiles <= kChipCUs && keys >= 8192 && tiles * keys >= 2 * kChipCUs * 1024)))
    return attend_rows_blocks(head_dim);
  return !wide && some && blocks * keys >= 3 << 18 ? 2 : 1;
}

// Shares of the keys, of `base` workgroups without any.  A second share costs a launch that joins (3 us, and as much on the host)
// and every workgroup a start of several dependent loads, so: none up to 1280 keys (8 KV heads, one context: 1000 keys 10.1 us
// whole, 9.5 shared; 2000 keys 15.0 and 9.7); up to a workgroup on each compute unit shares of 128 keys, up to two of 512 (16000
// keys: 13.8 us in 128 workgroups, 12.1 in 256, 12.8 in 512), beyond that, where contexts are uneven and the last ones
// would run alone, of 2048 (64 contexts of up to 8192 keys: 109 us in 512 workgroups, 89 in 2048; of up to 4000: 41 and 44), but not
// for contexts of several workgroups, whose results are more to join (64 queries, 32000 keys: 59 us in 960 workgroups, 53 in 512).
constexpr int kWholeKeys = 1280;
struct ShareRule {
  int workgroups, keys;                      // up to so many in all, of so many keys at least
  bool one_tile;                             // only where contexts are a workgroup's
};
constexpr ShareRule kShareRules[] = {{kChipCUs, 128, false}, {2 * kChipCUs, 512, false}, {8 * kChipCUs, 2048, true}};
static int key_shares(int64_t base, int64_t keys, bool one_tile) {
  if (base <= 0 || keys <= kWholeKeys) return 1;
  int64_t n = 1;
  for (const ShareRule& r : kShareRules)
    if (one_tile || !r.one_tile) n = std::max(n, std::min(r.workgroups / base, keys / r.keys));
  return (int)n;
}

static int64_t row_bytes(int head_dim) { return 4 * (head_dim + 2); }       // of a row's share: see AttendArgs::part

AttendPlan plan_attend(int n_q, int n_kv, int head_dim, int n_seq, int total_q, int max_q, int max_kv) {
  AttendPlan p;
  const int64_t group = n_q / n_kv, rows = std::max<int64_t>((int64_t)max_q * group, 1), all_rows = (int64_t)total_q * group;
  // tiles of `size` rows of all contexts and KV heads, about
  auto tiles_of = [&](int64_t size) { return n_kv * std::max<int64_t>(n_seq, (all_rows + size - 1) / size); };
  const int64_t many = 16 * attend_rows_blocks(head_dim);
  // Among contexts of other sizes than the longest's, single tokens mostly, wide workgroups are wasted: 512 queries on 512 keys and 63 times
  // one on 2000, 14 heads of 64 over 2, 15 us with 1 block, 20 with 2, 37 in kv4_prompt.hip; 32 heads of 128 over 8, 2048 queries twice and
  // 200 times one 208, 184, 206, 8192 queries and 255 times one 999, 774, 821, and 63 times one 904, 671, 606.
  const bool even = 2 * (int64_t)total_q >= (int64_t)n_seq * max_q;
  const bool filled = 4 * rows >= 3 * ((rows + many - 1) / many) * many && all_rows >= (even ? 3 * many / 4 : 8 * many) * n_seq;
  const bool some = rows > 16 && (even || all_rows >= 64 * (int64_t)n_seq);
  p.row_blocks = row_blocks(head_dim, tiles_of(16), max_kv, tiles_of(many), some, filled);
  p.paired = p.row_blocks == 1 && rows <= kPairedRows;
  const int64_t size = 16 * p.row_blocks;
  // a place a tile: contexts of very different sizes then leave next to none empty (8192 queries and 255 times one: 774 us; with places
  // for the longest in every context 1760)
  p.flat = rows > size;
  p.n_slots = (int)(p.flat ? all_rows / size + n_seq : n_seq);
  p.n_split = key_shares(tiles_of(size), max_kv, !p.flat && p.row_blocks <= 2);
  p.workspace = p.n_split > 1 ? p.n_split * ((int64_t)total_q * n_q) * row_bytes(head_dim) : 0;
  return p;
}

// Of calls of up to these sizes.  By a rule there are n <= workgroups / base shares, and base is at least n_kv, and at least rows / size
// where workgroups have `size` rows: n * rows is at most workgroups / n_kv * rows, keys / r.keys * rows, and workgroups * size.  Each of
// them, and with them the result, grows with the sizes or stays.
int64_t attend_workspace_bound(int n_q, int n_kv, int head_dim, int total_q, int max_kv) {
  if (max_kv <= kWholeKeys) return 0;
  const int64_t rows = std::min<int64_t>((int64_t)total_q * n_q, INT_MAX);      // calls have no more
  const int few = head_dim == 256 ? 16 : 32, many = head_dim == 256 ? 16 : 16 * attend_rows_blocks(head_dim);     // see row_blocks
  int64_t most = 0;
  for (const ShareRule& r : kShareRules) {
    const int64_t n = std::min(r.workgroups / n_kv, max_kv / r.keys);
    if (n > 1) most = std::max(most, std::min(n * rows, (int64_t)r.workgroups * (r.one_tile ? few : many)));
  }
  return most * row_bytes(head_dim);
}

template <int HD>
static void launch_hd(const AttendArgs& a, const AttendPlan& plan, hipStream_t stream) {
  const dim3 grid = attend_grid(a);
  if (plan.row_blocks > 2) {
    launch_attend_rows(a, HD, stream);
  } else if (plan.row_blocks == 1) {
    if (plan.paired) hipLaunchKernelGGL((attend_kernel<HD, 1, true>), grid, dim3(64 * kFewWaves), 0, stream, a);
    else             hipLaunchKernelGGL((attend_kernel<HD, 1, false>), grid, dim3(64 * kFewWaves), 0, stream, a);
  } else if constexpr (HD <= 128) {
    hipLaunchKernelGGL((attend_kernel<HD, 2, false>), grid, dim3(64 * kFewWaves), 0, stream, a);
  }
  if (a.n_split > 1) {
    const int64_t n_row = (int64_t)a.total_q * a.n_q;
    if (a.n_split <= 4) hipLaunchKernelGGL((attend_join_kernel<HD, 4>), dim3((unsigned)((n_row + 3) / 4)), dim3(256), 0, stream, a);
    else                hipLaunchKernelGGL((attend_join_kernel<HD, 16>), dim3((unsigned)n_row), dim3(256), 0, stream, a);
  }
}

hipError_t launch_attend(const AttendArgs& a, int head_dim, const AttendPlan& plan, hipStream_t stream) {
  if (a.total_q <= 0 || a.n_seq <= 0) return hipSuccess;
  switch (head_dim) {
    case 64: launch_hd<64>(a, plan, stream); break;
    case 128: launch_hd<128>(a, plan, stream); break;
    case 256: launch_hd<256>(a, plan, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hc
