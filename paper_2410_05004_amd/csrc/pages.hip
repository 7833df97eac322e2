// Pages of a cache as a whole: contexts that share them (forks), and packing them to the front of their pools.
#include "pages.h"

namespace hc {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// ---- fork -----------------------------------------------------------------------------------
// blockIdx: (piece of a page, fork, share of the pools); the share behind the last writes the children's table rows.
// A child's row is its parent's for the full blocks, its own page for a part-filled last one, -1 behind it; of that
// page the tokens in use are copied.  Parents' rows and children's are different rows, so no order matters.
// Bound: latency for a few forks (the parent's table entry, then the page: 8 forks in 32 layers 6 us), memory for many (64 forks of 17 KiB
// pages in 80 layers 33 us, 5.4 TB/s).  A workgroup looks the page up once and copies the same piece of it, up to 20 KiB, in every
// so-many-th pool (with a piece of 16 KiB of one pool a workgroup those 64 took 62 us: looking up, and a second piece of 1 KiB).
constexpr int kForkWords = kForkPiece / 256;   // of a thread
__global__ __launch_bounds__(256) void fork_kernel(const ForkArgs a) {
  const int f = blockIdx.y, share = blockIdx.z;
  const int n_tok = a.n_tok[f], whole = n_tok >> a.block_shift, rest = n_tok & ((1 << a.block_shift) - 1);
  const int32_t* parent = a.tables + (size_t)a.from[f] * a.max_blocks;
  // the page to copy: valid, and not the one that it is to be copied into
  int last = 0;
  bool ok = true;
  if (rest) {
    last = parent[whole];
    ok = last >= 0 && last < a.num_pages && last != a.page[f];
  }
  if (share == a.shares) {
    if (blockIdx.x) return;
    int32_t* child = a.tables + (size_t)a.to[f] * a.max_blocks;
    for (int b = threadIdx.x; b < a.max_blocks; b += 256)
      child[b] = b < whole ? parent[b] : b == whole && rest && ok ? a.page[f] : -1;
    if (!ok && threadIdx.x == 0) atomicOr(a.err, HC_DEV_BAD_PAGE);
    return;
  }
  if (!rest || !ok) return;
  for (int kind = 0; kind < 2; ++kind) {
    const int begin = kind ? a.pools.first4 : 0, end = kind ? a.pools.n_pools : a.pools.first4;
    if (begin + share >= end) continue;
    const PageShape& s = a.pools.shape[kind];
    const int run = ((rest + (1 << s.unit_shift) - 1) >> s.unit_shift) * s.unit, total = s.runs * run;
    int at[kForkWords];
    bool in[kForkWords];
#pragma unroll
    for (int u = 0; u < kForkWords; ++u) {
      const int i = blockIdx.x * kForkWords * 256 + u * 256 + threadIdx.x;
      in[u] = i < total;
      at[u] = run == s.stride ? i : i / run * s.stride + i % run;
    }
    const size_t from = (size_t)last * s.words, to = (size_t)a.page[f] * s.words;
    for (int pool = begin + share; pool < end; pool += a.shares) {
      u32x4* base = static_cast<u32x4*>(a.pools.pool[pool]);
      u32x4 v[kForkWords];
#pragma unroll
      for (int u = 0; u < kForkWords; ++u)
        if (in[u]) v[u] = __builtin_nontemporal_load(base + from + at[u]);
#pragma unroll
      for (int u = 0; u < kForkWords; ++u)
        if (in[u]) __builtin_nontemporal_store(v[u], base + to + at[u]);
    }
  }
}

hipError_t launch_fork(const ForkArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(fork_kernel, dim3(a.pieces, a.n_fork, a.shares + (a.with_tables ? 1 : 0)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

// ---- compact --------------------------------------------------------------------------------
// Live pages (those that a table names) are to be pages 0 .. live - 1: a live page there stays, the others move, in their
// order, to the free pages among them, in theirs.  One workgroup works the plan out: a bit a page in LDS, set from the
// tables, then ranks by counting bits: page p's rank among the live is prefix(p); free pages before p are p - prefix(p).
// The map and the pairs are written by all of it in one pass over the pages.
// Bound: one compute unit's reads of the tables and writes of the map, and latency: 500 pages 3.8 us, 2048 4.9, 2^17 57, 2^20 720 (with as
// many parts as threads 1550: a page's rank is a sum over half a part's words).
constexpr int kPlanThreads = 1024, kPlanParts = 4096;            // live pages are counted by parts of the bits
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(const CompactArgs a) {
  extern __shared__ uint32_t s_bits[];
  __shared__ int s_before[kPlanParts], s_wave[kPlanThreads / 64];
  const int tid = threadIdx.x, n = a.num_pages, words = (n + 31) >> 5;
  const int per = (words + kPlanParts - 1) / kPlanParts;         // words of a part
  for (int i = tid; i < words; i += kPlanThreads) s_bits[i] = 0;
  __syncthreads();
  bool bad = false;
  for (int64_t i0 = tid; i0 < a.entries; i0 += 8 * kPlanThreads) {
    int p[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = i0 + (int64_t)u * kPlanThreads;
      p[u] = i < a.entries ? a.tables_in[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (p[u] >= n) bad = true;
      else if (p[u] >= 0) atomicOr(&s_bits[p[u] >> 5], 1u << (p[u] & 31));
    }
  }
  if (bad) atomicOr(a.err, HC_DEV_BAD_PAGE);
  __syncthreads();
  constexpr int kMine = kPlanParts / kPlanThreads;
  int part[kMine], mine = 0;
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    part[u] = mine;
    for (int i = 0; i < per; ++i) {
      const int w = (tid * kMine + u) * per + i;
      if (w < words) mine += __popc(s_bits[w]);
    }
  }
  int sum = mine;                                                // inclusive over the wave, then over the waves
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(sum, d);
    if ((tid & 63) >= d) sum += o;
  }
  if ((tid & 63) == 63) s_wave[tid >> 6] = sum;
  __syncthreads();
  int live = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    if (i < (tid >> 6)) sum += s_wave[i];
    live += s_wave[i];
  }
#pragma unroll
  for (int u = 0; u < kMine; ++u) s_before[tid * kMine + u] = sum - mine + part[u];
  __syncthreads();
  auto prefix = [&](int p) __attribute__((always_inline)) {      // live pages before p
    const int w = p >> 5, t = w / per;
    int c = s_before[t];
    for (int i = t * per; i < w; ++i) c += __popc(s_bits[i]);
    return c + (p & 31 ? __popc(s_bits[w] & ((1u << (p & 31)) - 1)) : 0);
  };
  const int stay = live < n ? prefix(live) : n, moves = live - stay;
  int32_t* map = a.plan + 2;
  int32_t* pairs = map + n;
  if (tid == 0) { a.plan[0] = live; a.plan[1] = moves; }
  for (int p = tid; p < n; p += kPlanThreads) {
    const bool is = s_bits[p >> 5] >> (p & 31) & 1;
    const int before = prefix(p);
    if (is && p >= live) pairs[2 * (before - stay)] = p;
    else {
      map[p] = is ? p : -1;
      if (!is && p < live) pairs[2 * (p - before) + 1] = p;
    }
  }
  __syncthreads();                                               // the pairs are read by others of the workgroup than wrote them
  for (int i = tid; i < moves; i += kPlanThreads) map[pairs[2 * i]] = pairs[2 * i + 1];
}

// Pages to their new places, in every pool, in steps of up to 20 KiB, equal ones of a page, and the tables through the map.  The launch does
// not know how many there are.  Bound: memory: 32 layers' bf16 pages of 64 KiB, 454 moves, 356 us, 5.3 TB/s read and written (a large copy: 4.9);
// 8 layers' 4-bit pages of 17 KiB, 34 MB, 6 to 7 us (in steps of 16 KiB, every other one of 1 KiB, 9 to 10).
constexpr int kMovePiece = 5 * 256;        // words of a step at most
__global__ __launch_bounds__(256) void compact_move_kernel(const CompactArgs a) {
  const int32_t* map = a.plan + 2;
  const int32_t* pairs = map + a.num_pages;
  if (a.with_tables)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.entries; i += (int64_t)gridDim.x * 256) {
      const int p = a.tables_in[i];
      a.tables_out[i] = p >= 0 && p < a.num_pages ? map[p] : -1;
    }
  const int moves = a.plan[1];
  for (int kind = 0; kind < 2; ++kind) {
    const int first = kind ? a.pools.first4 : 0, n_pools = (kind ? a.pools.n_pools : a.pools.first4) - first;
    if (n_pools <= 0) continue;
    const int words = a.pools.shape[kind].words, pieces = (words + kMovePiece - 1) / kMovePiece, length = (words + pieces - 1) / pieces;
    const int64_t items = (int64_t)moves * n_pools * pieces;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
      const int64_t pair = it / pieces;
      const int piece = (int)(it - pair * pieces), pool = (int)(pair % n_pools), move = (int)(pair / n_pools);
      u32x4* base = static_cast<u32x4*>(a.pools.pool[first + pool]);
      const u32x4* from = base + (size_t)pairs[2 * move] * words;
      u32x4* to = base + (size_t)pairs[2 * move + 1] * words;
      const int i0 = piece * length + threadIdx.x, end = piece * length + length < words ? piece * length + length : words;
      u32x4 v[kMovePiece / 256];
#pragma unroll
      for (int u = 0; u < kMovePiece / 256; ++u)
        if (i0 + u * 256 < end) v[u] = __builtin_nontemporal_load(from + i0 + u * 256);
#pragma unroll
      for (int u = 0; u < kMovePiece / 256; ++u)
        if (i0 + u * 256 < end) __builtin_nontemporal_store(v[u], to + i0 + u * 256);
    }
  }
}

hipError_t launch_compact_plan(const CompactArgs& a, hipStream_t stream) {
  const int bytes = (a.num_pages + 31) / 32 * 4;
  if (bytes > 32 * 1024) {               // more than a launch may have unasked, with what the kernel has beside it
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(compact_plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kMaxCompactPages / 8);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), bytes, stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_move(const CompactArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(compact_move_kernel, dim3(8 * kChipCUs), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace hc
