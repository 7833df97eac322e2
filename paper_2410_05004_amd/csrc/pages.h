// Forking contexts and compacting the pages of a cache: what the entry points and the kernels share.
#pragma once

#include "hcache_internal.h"

namespace hc {

constexpr int kForksPerLaunch = 64;
constexpr int kForkPiece = 5 * 256;       // 16-byte words of a page that a workgroup copies
constexpr int kPoolsPerLaunch = 128;      // pools (a layer's bf16 or 4-bit one) per launch
constexpr int kMaxCompactPages = 1 << 20; // one bit each in a compute unit's LDS

// A page of a pool, `words` 16-byte words: what a fork copies of it are `runs` runs, `stride` words apart, of `unit` words for every
// 2^unit_shift tokens begun (bf16: K and V; 4 bits: the KV heads).
struct PageShape {
  int32_t words, runs, stride, unit, unit_shift;
};
struct PoolList {
  void* pool[kPoolsPerLaunch];
  PageShape shape[2];                     // of the pools before `first4`, and of the others
  int32_t n_pools, first4;
};

struct ForkArgs {
  PoolList pools;
  int32_t from[kForksPerLaunch], to[kForksPerLaunch], n_tok[kForksPerLaunch], page[kForksPerLaunch];
  int32_t* tables;
  int32_t* err;
  int64_t num_pages;
  int32_t n_fork, max_blocks, block_shift, with_tables;
  int32_t pieces, shares;                 // of a page (kForkPiece words); of the pools
};
hipError_t launch_fork(const ForkArgs& a, hipStream_t stream);

struct CompactArgs {
  PoolList pools;
  const int32_t* tables_in;
  int32_t* tables_out;
  int32_t* plan;                          // live pages, moves, new place of every page (-1: freed), (from, to) of the moves
  int32_t* err;
  int64_t entries;
  int32_t num_pages, with_tables;
};
hipError_t launch_compact_plan(const CompactArgs& a, hipStream_t stream);
hipError_t launch_compact_move(const CompactArgs& a, hipStream_t stream);

}  // namespace hc
