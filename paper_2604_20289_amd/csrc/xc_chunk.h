// Chunks of new tokens over the paged cache and what it keeps: the kernels'
// arguments and launchers.
#pragma once

#include "xc_chunk_plan.h"
#include "xc_pool.h"

namespace xc {

// What xc_chunk_set leaves to the sums of weights: units and tiles, or, where
// all sequences have few rows, runs.
struct WeightArgs {
  PageBuf buf;
  const int* tables;
  const ChunkSeq* seqs;
  ChunkMask mask;
  int q_heads, group;  // group: query heads per key head
  unsigned by_group;   // 2^32 / group rounded up, 0 for 1: r / group is the high half of r * by_group
  const WeightUnit* units;
  const WeightTile* tiles;
  int n_units, n_long, n_tiles;
  float* parts;        // [part][key head][kWeightKeys] (float32 pools: kWeightKeysF32)
  const WeightFew* runs;
  const WeightInfo* infos;
  int n_runs, n_groups;
  const void* q;       // [rows][q_ld]
  long long q_ld;
  float scale;         // of q . k, in log2 units
  const float* lse;    // [rows][q_heads]
  float decay;
  float* weights;      // [sequence][ld]
  long long ld;
};

// A sequence that gives tokens up.
struct EvictSeq {
  int number;        // row of weights and kept
  int first, tokens;
  int keep;          // < tokens; -1: all of them, only listed
  int from, to;      // its old and new page table begin at tables[from], tables[to]
  int at;            // its kept tokens' places begin at src[at]
  int replaced;      // some of its kept pages are other ones now
};
struct EvictArgs {
  EvictSeq* seqs;
  int* tables;
  int* src;    // places (page * page tokens + row) of the kept tokens
  int* stays;  // [n] of its first tokens, all kept
  int n, sinks, recent;
  float* weights;  // [n][ld]
  long long ld;
  int* kept;       // [n][kept_ld], may be null
  long long kept_ld;
};

hipError_t launch_weights(int dtype, const WeightArgs& a, hipStream_t st);
// What fits into a kernel's arguments.
struct Little {
  static constexpr size_t kMost = 3584;
  alignas(16) char bytes[kMost];
};
// whole: the first block; of the sequences that shrink, most_tokens before and
// `most` kept; little: what seqs and, as far behind them, tables are to hold (null: they do)
hipError_t launch_evict(const EvictArgs& a, const Little* little, const PageBuf& whole, int esz, int n_blocks,
                        long long block_bytes, int most_tokens, int most, hipStream_t st);

}  // namespace xc
