// Attention of many rows over the 4-bit cache: prompts on histories.  The mathematics and the matrix ops' operands are
// those of kv4_attend.hip; here a decoded key or value serves 128 * NB rows of a workgroup instead of 16 * NB.
#include "kv4_device.h"

namespace hc {

// A workgroup takes 128 * NB rows, 32 * NB to a wave, and a share of the keys in tiles of 64.  Each wave decodes a quarter of
// a tile into LDS, as the operands of v_mfma_f32_32x32x16 (1 KiB a fragment, 16 bytes a lane in lane order), while all of
// them work on the tile before; the bytes of the tile behind are on their way to registers meanwhile.
// Bound: issue: 8 contexts of up to 2048 queries on 4096 keys, 40 heads of 128, 454 GFLOP, 502 to 550 us (0.83 to 0.90 PFLOP/s, by
// card; a large product of the library's reaches 1.21), matrix instructions 45 % of the cycles and vector ones 52: of a wave's 32 rows and 64 keys, 32 matrix
// instructions of 32 cycles, the softmax's 2048 exponentials and its maxima and sums beside them, and a quarter of the tile's decoding.
// Weights are rounded to bf16, 2^-8 relative at most (outputs are off by 0.0023 in norm, of which their own rounding makes 0.0017); the rest of
// them in a second product: 846 us, so 1072 with it (8 times 2048 queries, 40 heads, up to 4096 keys).
// 32 x 32 products take half the issue slots of 16 x 16 ones; a second workgroup on the compute unit fills the barriers.
// As K's rows lane (l32, half) takes key l32 and, in step j, channels (2 * (j / n) + half) * HD / 4 + j % n * 8 .. + 7, n = HD / 32; as
// V^T's rows channels of slice l32 % 16, the even or the odd one of pair c.
template <int HD, int NB>       // NB: blocks of 32 rows of a wave
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(const AttendArgs a) {
  constexpr int kSteps = HD / 16, kBlocks = HD / 32, kTile = 64, kWaves = 4;       // matrix ops along the channels; blocks of 32 channels of the result
  __shared__ u32x4 s_k[2][2][kSteps][64], s_v[2][2][2][kBlocks][64];
  __shared__ int s_range[kWaves][4], s_nan[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, q4 = lane >> 4, l32 = lane & 31, half = lane >> 5;
  const int split = blockIdx.x % a.n_split, kvh = blockIdx.x / a.n_split;
  const Task task(a, 32 * NB * kWaves);
  const int seq = task.seq, q0 = task.q0, n_rows = task.n_rows;
  const int64_t room = (int64_t)a.max_blocks << a.block_shift, most = room < kMaxKeys ? room : kMaxKeys;
  int keys = uniform(a.kv_lens)[seq];
  if (keys > most || keys < 0) {
    if (threadIdx.x == 0) atomicOr(a.err, HC_DEV_BAD_POSITION);
    keys = keys < 0 ? 0 : (int)most;
  }
  if (task.tile < 0) return;                         // not before the count is asked for: both are on their way together
  Places places(a, seq, kvh, sub_bytes(HD));
  bool bad_page = false;

  for (int tile_of_rows = task.tile; tile_of_rows >= 0; tile_of_rows -= task.step) {
    const int block0 = (tile_of_rows * kWaves + wave) * NB;                // this wave's first block of rows
    auto row_of = [&](int nb) __attribute__((always_inline)) {
      const int r = (block0 + nb) * 32 + l32;
      return r < n_rows ? r : n_rows - 1;
    };
    int lo[NB], hi[NB];
    int begin = 0x7fffffff, end = 0, all_lo = 0, all_hi = 0x7fffffff;
    bf16x8 q[NB][kSteps];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = row_of(nb), qi = r / a.group, pos = a.positions[q0 + qi];
      hi[nb] = pos < keys - 1 ? pos : keys - 1;
      lo[nb] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
      const bool sees = hi[nb] >= lo[nb];
      begin = min_of(begin, sees ? lo[nb] : 0x7fffffff);
      end = max_of(end, sees ? hi[nb] + 1 : 0);
      all_lo = max_of(all_lo, lo[nb]);
      all_hi = min_of(all_hi, hi[nb]);
      const uint16_t* from = a.q + (q0 + qi) * a.q_stride + (kvh * a.group + r - qi * a.group) * HD + half * (HD / 4);
#pragma unroll
      for (int j = 0; j < kSteps; ++j) q[nb][j] = *reinterpret_cast<const bf16x8*>(from + j / kBlocks * (HD / 2) + j % kBlocks * 8);
    }
    begin = __builtin_amdgcn_readfirstlane(across_32(begin, min_of));
    end = __builtin_amdgcn_readfirstlane(across_32(end, max_of));
    all_lo = __builtin_amdgcn_readfirstlane(across_32(all_lo, max_of));
    all_hi = __builtin_amdgcn_readfirstlane(across_32(all_hi, min_of));
    if (lane == 0) { s_range[wave][0] = begin; s_range[wave][1] = end; s_range[wave][2] = all_lo; s_range[wave][3] = all_hi; }
    __syncthreads();
    int wg_begin = begin, wg_end = end, wg_lo = all_lo, wg_hi = all_hi;   // of the workgroup's rows
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      wg_begin = min_of(wg_begin, s_range[i][0]);
      wg_end = max_of(wg_end, s_range[i][1]);
      wg_lo = max_of(wg_lo, s_range[i][2]);
      wg_hi = min_of(wg_hi, s_range[i][3]);
    }
    wg_begin = __builtin_amdgcn_readfirstlane(wg_begin);
    wg_end = __builtin_amdgcn_readfirstlane(wg_end);
    wg_lo = __builtin_amdgcn_readfirstlane(wg_lo);
    wg_hi = __builtin_amdgcn_readfirstlane(wg_hi);
    // ---- this workgroup's share of the keys, in tiles
    const int first = wg_begin < wg_end ? wg_begin / kTile : 0;
    const int n_all = wg_begin < wg_end ? (wg_end + kTile - 1) / kTile - first : 0;
    const int share = (n_all + a.n_split - 1) / a.n_split;
    const int from_tile = first + split * share, to_tile = min_of(from_tile + share, first + n_all);

    f32x16 o[NB][kBlocks];
    float top[NB], limit[NB], sum[NB];               // weights are 2^(score - top); limit: how far a score may be above it, nothing before the first key
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      limit[nb] = kNegInf;
      top[nb] = sum[nb] = 0.f;
#pragma unroll
      for (int c = 0; c < kBlocks; ++c) o[nb][c] = f32x16{};
    }

    // this wave's 16 keys of a tile; a round of places has the runs of 16 tiles
    constexpr int kRound = 64 / kWaves, kRuns = (1 << kWaves) - 1;
    RawK<HD> rk;
    RawV<HD> rv;
    auto find = [&](int tile) __attribute__((always_inline)) {        // this wave's run of a tile; tiles come in order
      const int at = (tile - from_tile) % kRound * kWaves;
      if (at == 0) {
        places.settle(tile * kTile + 16 * lane);
        places.look_up((tile + kRound) * kTile + 16 * lane);
      }
      return places.of(at + wave);
    };
    auto missing = [&](int tile) __attribute__((always_inline)) { return ~(int)(places.there >> (tile - from_tile) % kRound * kWaves) & kRuns; };   // runs without a page
    auto is_edge = [&](int tile, int gone) __attribute__((always_inline)) { return tile * kTile < wg_lo || tile * kTile + kTile - 1 > wg_hi || gone; };
    auto hide = [&](int buf, int tile, int gone) __attribute__((always_inline)) {
      const bool nan_value = only_seen<HD>(rv, tile * kTile + 16 * wave + 4 * q4, wg_begin, wg_end, gone >> wave & 1);
      if (__any(nan_value)) s_nan[buf] = tile + 1;
    };
    auto decode_keys = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        const float ks = rk.scale(l16, q4, j);
        u32x4 k;
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = decode2(rk.w[j], ks, i);
        s_k[buf][wave >> 1][kBlocks * (q4 >> 1) + j][(q4 & 1) * 32 + (wave & 1) * 16 + l16] = k;
      }
    };
    auto decode_values = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        uint32_t c[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int byte = t * (HD / 32) + i;
          c[t] = decode2(rv.w[byte >> 2], scale_of(rv.scales, t), byte & 3);
        }
        // half a lane's part of a fragment: four of its eight keys; the even channels in rows 0 .. 15 of 32, the odd behind
        u32x4* to = &s_v[buf][wave >> 1][wave & 1][i][(q4 & 1) * 32 + l16];
        u32x2* even = reinterpret_cast<u32x2*>(to) + (q4 >> 1);
        u32x2* odd = reinterpret_cast<u32x2*>(to + 16) + (q4 >> 1);
        *even = u32x2{__builtin_amdgcn_perm(c[1], c[0], 0x05040100), __builtin_amdgcn_perm(c[3], c[2], 0x05040100)};
        *odd = u32x2{__builtin_amdgcn_perm(c[1], c[0], 0x07060302), __builtin_amdgcn_perm(c[3], c[2], 0x07060302)};
      }
    };

    // Scores of 32 keys, register v being key 8 * (v / 4) + 4 * half + v % 4, and how far a lane's are above the top at most.
    struct Scores {
      f32x16 x[NB];
      float most[NB];
    };
    // Operands of 32 keys, read together: the compiler by itself reads each into the registers of the one before, right before its
    // use, and waits (8 contexts of 2048 queries on up to 4096 keys, 40 heads of 128, 846 us, so 864; one of 501 on 8692, 32 heads over 8, 91.6 and
    // 92.8).  At 64 channels 10 registers go to scratch for it, 1 without: as fast either way (4 heads, 64 contexts of 512 on up to 4000 177 and 178).
    struct KeyParts {
      bf16x8 k[kSteps];
    };
    struct ValueParts {
      bf16x8 v[2][kBlocks];
    };
    auto read_keys = [&](KeyParts& f, int buf, int pair) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) f.k[j] = __builtin_bit_cast(bf16x8, s_k[buf][pair][j][lane]);
      __builtin_amdgcn_sched_barrier(6);             // vector and scalar instructions may pass, the products and the next reads may not
    };
    auto read_values = [&](ValueParts& f, int buf, int pair) __attribute__((always_inline)) {
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) f.v[m][c] = __builtin_bit_cast(bf16x8, s_v[buf][pair][m][c][lane]);
    };
    auto products = [&](Scores& s, const KeyParts& f) __attribute__((always_inline)) {       // S^T = K Q^T
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s.x[nb] = f32x16{};
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s.x[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.k[j], q[nb][j], s.x[nb], 0, 0, 0);
    };
    auto most_of = [&](Scores& s) __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float m = larger(s.x[nb][0], s.x[nb][1]);
#pragma unroll
        for (int v = 2; v < 16; v += 2) m = larger(larger(m, s.x[nb][v]), s.x[nb][v + 1]);
        s.most[nb] = m;
      }
    };
    auto above_top = [&](Scores& s) __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int v = 0; v < 16; ++v) s.x[nb][v] = __builtin_fmaf(s.x[nb][v], a.scale_log2, -top[nb]);
      most_of(s);
    };
    auto weights = [&](bf16x8 (&w)[NB][2], const Scores& s) __attribute__((always_inline)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float e = __builtin_amdgcn_exp2f(s.x[nb][v]);
          sum[nb] += e;
          w[nb][v >> 3][v & 7] = (__bf16)e;
        }
    };
    auto add_values = [&](const bf16x8 (&w)[NB][2], const ValueParts& f) __attribute__((always_inline)) {   // O^T += V^T W^T
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) o[nb][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v[m][c], w[nb][m], o[nb][c], 0, 0, 0);
    };
    // What new scores ask for now and then: masks, NaN among the values, a higher top.
    auto settle = [&](Scores& s, int tile, int buf, int pair, int gone) __attribute__((always_inline)) {
      const int key0 = tile * kTile + 32 * pair;
      const int gone2 = gone >> (2 * pair) & 3;
      if (key0 < all_lo || key0 + 31 > all_hi || gone2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if ((gone2 >> h & 1) && key0 + 16 * h < end && key0 + 16 * h + 15 >= begin) bad_page = true;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = key0 + 8 * (v >> 2) + 4 * half + (v & 3);
          const bool out = gone2 >> (v >> 3) & 1;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) s.x[nb][v] = out || key < lo[nb] || key > hi[nb] ? kNegInf : s.x[nb][v];
        }
        most_of(s);
      }
      bool high = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) high |= s.most[nb] > limit[nb];
      if (__any(high)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float rise = across_halves(s.most[nb], [](float p, float r) { return fmaxf(p, r); });
          // rows without a key yet keep their top, of whatever height: their sums are zero
          const bool fresh = limit[nb] == kNegInf;
          const float by = rise == kNegInf ? 0.f : fresh ? rise : fmaxf(rise, 0.f);
          limit[nb] = rise == kNegInf ? limit[nb] : kTopSlack;
          top[nb] += by;
          const float shrink = fresh ? 1.f : __builtin_amdgcn_exp2f(-by);
          sum[nb] *= shrink;
#pragma unroll
          for (int c = 0; c < kBlocks; ++c) o[nb][c] *= shrink;
          s.x[nb] -= by;
        }
      }
      if (is_edge(tile, gone) && s_nan[buf] == tile + 1) {       // taken out of the tile, given to the rows that see it here
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            // registers 4 * u + i and 8 + 4 * u + i, i < 4, are channels of slices 8 * u + 4 * half + i, of one group of 32
            const float poison = nan_values<HD>(places, key0, 32, lo[nb], hi[nb], (8 * u + 4 * half) * HD / 512);
#pragma unroll
            for (int c = 0; c < kBlocks; ++c)
#pragma unroll
              for (int x = 0; x < 8; ++x) o[nb][c][8 * (x >> 2) + 4 * u + (x & 3)] += poison;
          }
      }
    };

    // Steps of 32 keys.  A step takes the first products of the 32 keys behind with the weights of its own, then its own second
    // products; the values of the tile behind are decoded in the first step, the keys of the one after that in the last.
    if (threadIdx.x < 2) s_nan[threadIdx.x] = 0;     // 1 + the last tile of this buffer with NaN among its values
    __syncthreads();
    if (from_tile < to_tile) {
      // runs without a page: of the tile worked on, the one whose values are in registers, and the one whose keys are (behind
      // the last tile: bytes of some page, not used)
      int gone = 0, gone_v = 0, gone_k = 0;
      Scores s0, s1;
      bf16x8 w[NB][2];
      places.look_up(from_tile * kTile + 16 * lane);
      const uint8_t* at = find(from_tile);
      gone = missing(from_tile);
      rk.load(at, l16, q4);
      rv.load(at, l16, q4);
      if (is_edge(from_tile, gone)) hide(0, from_tile, gone);
      decode_keys(0);
      decode_values(0);
      at = find(from_tile + 1);
      gone_v = gone_k = missing(from_tile + 1);
      rk.load(at, l16, q4);
      rv.load(at, l16, q4);
      decode_keys(1);
      at = find(from_tile + 2);
      gone_k = missing(from_tile + 2);
      rk.load(at, l16, q4);
      __syncthreads();
      KeyParts k0;
      read_keys(k0, 0, 0);
      products(s0, k0);
      above_top(s0);
      for (int tile = from_tile; tile < to_tile; ++tile) {
        const int buf = (tile - from_tile) & 1;
        if (is_edge(tile + 1, gone_v)) hide(buf ^ 1, tile + 1, gone_v);
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
          const bool last = pair == 1;
          Scores& now = pair & 1 ? s1 : s0;
          Scores& next = pair & 1 ? s0 : s1;
          if (last) __syncthreads();                 // the next tile's values are there, and this one's keys are not needed any more
          settle(now, tile, buf, pair, gone);
          KeyParts k;
          ValueParts v;
          read_keys(k, last ? buf ^ 1 : buf, last ? 0 : pair + 1);
          products(next, k);
          read_values(v, buf, pair);
          weights(w, now);
          add_values(w, v);
          above_top(next);
          if (pair == 0) {
            decode_values(buf ^ 1);
            rv.load(at, l16, q4);
          }
          if (last) {
            decode_keys(buf);
            at = find(tile + 3);
            rk.load(at, l16, q4);
          }
        }
        gone = gone_v;
        gone_v = gone_k;
        gone_k = missing(tile + 3);
        __syncthreads();                             // the keys behind are there, and this tile's values are not needed any more
      }
    }

    // ---- results; places behind the last row have computed that row too and store the same
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float total = across_halves(sum[nb], [](float p, float r) { return p + r; });
      if ((block0 + nb) * 32 >= n_rows) continue;
      const int r = row_of(nb), qi = r / a.group, head = kvh * a.group + r - qi * a.group;
      const int64_t tok = q0 + qi, row = tok * a.n_q + head;
      const int64_t n_row = (int64_t)a.total_q * a.n_q;
      const float norm = a.n_split > 1 ? 1.f : total == 0.f ? 0.f : 1.f / total;
      // slice 8 * u + 4 * half + i: HD / 16 consecutive channels, 2 c + odd being register 8 * odd + 4 * u + i of block c
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = (8 * u + 4 * half + i) * (HD / 16);
#pragma unroll
          for (int c = 0; c < kBlocks; c += 2) {
            const f32x4 x = {o[nb][c][4 * u + i] * norm, o[nb][c][8 + 4 * u + i] * norm, o[nb][c + 1][4 * u + i] * norm, o[nb][c + 1][8 + 4 * u + i] * norm};
            if (a.n_split == 1) {
              u32x2 y;
              y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[0], x[1]}, bf16x2));
              y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2], x[3]}, bf16x2));
              *reinterpret_cast<u32x2*>(a.out + tok * a.out_stride + head * HD + at + 2 * c) = y;
            } else {
              *reinterpret_cast<f32x4*>(a.part + (split * n_row + row) * HD + at + 2 * c) = x;
            }
          }
        }
      if (a.n_split > 1)
        *reinterpret_cast<f32x2*>(a.part + a.n_split * n_row * HD + (split * n_row + row) * 2) = f32x2{limit[nb] == kNegInf ? kNegInf : top[nb], total};
      else if (a.lse)
        a.lse[row] = top[nb] * 0.69314718056f + __logf(total);
    }
  }
  if (bad_page && lane == 0) atomicOr(a.err, HC_DEV_BAD_PAGE);
}

// blocks of 32 rows of a wave: as many as leave room for two waves in a SIMD's registers, all but a few at 64 channels
constexpr int wave_blocks(int head_dim) { return head_dim == 64 ? 2 : 1; }

int attend_rows_blocks(int head_dim) { return 8 * wave_blocks(head_dim); }

void launch_attend_rows(const AttendArgs& a, int head_dim, hipStream_t stream) {
  const dim3 grid = attend_grid(a);
  if (head_dim == 64) hipLaunchKernelGGL((attend_rows_kernel<64, wave_blocks(64)>), grid, dim3(256), 0, stream, a);
  else                hipLaunchKernelGGL((attend_rows_kernel<128, wave_blocks(128)>), grid, dim3(256), 0, stream, a);
}

}  // namespace hc
