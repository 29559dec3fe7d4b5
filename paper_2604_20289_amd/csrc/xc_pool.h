// Internal declarations of the branching cache: its kernels' arguments and
// launchers, and what xc_seq_import needs to know of a model handle.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "xc_branch_plan.h"
#include "xc_chunk_plan.h"
#include "xc_pages.h"

struct xc_handle;

namespace xc {

// A block's page buffers: keys and values as [page][kv_heads][page tokens][D].
struct PageBuf {
  void* keys;
  void* values;
  int shift;     // log2 of the tokens per page
  int kv_heads;
  int D;
};

// The most page copies of one launch: they travel in its arguments (the few of
// a fork in a short form: the arguments of a launch are copied too).
constexpr int kCopyBatch = 300, kCopyBatchFew = 24;
template <int N>
struct CopyArgs {
  PageCopy c[N];
};
static_assert(sizeof(CopyArgs<kCopyBatch>) <= 3800, "kernel arguments");

// The most pages that one launch of the import fills.
constexpr int kImportPages = 900;
struct ImportArgs {
  int n_pages;
  int page[kImportPages];
};

// A model handle's rolling cache, for xc_seq_import.
struct HandleWindow {
  hipStream_t st;
  int device, dtype, n_blocks, heads, D, tokens;  // tokens: L of one chunk
  long long Lcap;
  const void* keys;    // [block][head][Lcap][D]
  const void* values;  // [block][head][D][Lcap]
  int chunks;          // kept past chunks, oldest first in slots
  std::vector<int> slots;
  bool sticky;
};
HandleWindow handle_window(const xc_handle* h);

// One rotary axis split: pairs [0, n0) follow axis 0, [n0, n0 + n1) axis 1,
// the rest axis 2; turns[pair] = theta^(-2i/d_a) / (2 pi).
struct RopeFreqs {
  int axes, n0, n1;
  double turns[64];
};

struct NormRopeArgs {
  const void* qkv;         // [rows][ld]: q heads, k heads, v heads
  long long ld;
  const float *gq, *gk;    // [D]
  const int* positions;    // [rows][axes], null: no rotation
  void* q_out;             // [rows][q_ld]
  long long q_ld;
  const int* place;        // [rows] page * page tokens + row
  int rows, q_heads;
  PageBuf buf;
  RopeFreqs freqs;
};

struct AttnArgs {
  const void* q;            // [rows][q_ld]
  void* out;                // [rows][out_ld]
  long long q_ld, out_ld;
  PageBuf buf;
  const int* tables;
  const AttnUnit* units;
  int n_units, n_long;      // the first n_long of them are the long ones
  int group;                // query heads per key head
  float scale;              // of q . k, in log2 units
  float* pieces;            // [slot][row - piece_row0][q_heads][D] unnormalised outputs
  float2* stats;            // [slot][row - piece_row0][q_heads] (running maximum in log2 units, sum)
  const OwnSlots* own;      // [rows] the slots of the row's own pieces; n = 0 and no shared slots: none
  int shared_slots;         // slots 0 .. shared_slots - 1 are pieces of every row
  int rows, q_heads;
  int piece_row0, piece_rows;  // the rows that have pieces: from piece_row0 to the last
  int n_slots;              // 0: no row has pieces
  int few;                  // bf16: units of at most kFewRows query rows, for branch_few_kernel
  // rows under a mask: units of their own in the place of `units`, else null
  const ChunkUnit* chunk_units;
  const ChunkSeq* chunk_seqs;
  ChunkMask mask;
  float* lse;               // [rows][q_heads] log-sum-exps, may be null
};


// n <= kCopyBatch copies, sources and destinations disjoint
hipError_t launch_page_copies(const PageCopy* copies, int n, const PageBuf& whole, int esz, int n_blocks,
                              long long block_bytes, hipStream_t st);
hipError_t launch_import(const ImportArgs& a, const HandleWindow& w, int slot, int chunk_token, int place0, int n_tokens,
                         const PageBuf& whole, long long block_elems, hipStream_t st);
hipError_t launch_norm_rope(int dtype, const NormRopeArgs& a, hipStream_t st);
hipError_t launch_branch_attention(int dtype, const AttnArgs& a, hipStream_t st);
// A sequence of a batch, as the expansion to rows reads it.
struct BatchSeq {
  int row0;      // its first batch row
  int at;        // the place, in its pages, of that row's token
  int table;     // where its page table begins
  OwnSlots own;
};
// place[row] and own[row] of every batch row from the n sequences (ascending
// row0; those without rows left out)
hipError_t launch_batch_rows(const int* tables, const BatchSeq* seqs, int n, int rows, int shift, int* place,
                             OwnSlots* own, hipStream_t st);

}  // namespace xc
