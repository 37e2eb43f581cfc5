// Batches of packed sequences: kernel arguments and the device functions that find a row's sequence, its slots and its pages
// (paged_append.hip, paged_attn.hip).  Lengths, prefix sums and page tables are read on the device and bounded there, so
// nothing that they hold leads an access out of the tensors.
#pragma once
#include "common.hpp"
#include "paged_plan.hpp"

namespace samkv {

struct RowsArg {  // samkv_rows with strides in bytes
  char* p;
  long long hs, rs;
};

struct BatchArg {
  int n_seq, n_rows, max_new, max_len;
  const int32_t* cu;     // null: every sequence has max_new rows
  const int32_t* len;    // null: prompts, a sequence is as long as its rows
  const int32_t* table;  // pages only
  int max_pages, n_pages, page_log2;
};

// Rows first .. first + n - 1 of the batch's tensors are the newest n of the sequence's len tokens.
struct SeqSpan {
  int first, n, len;
};
__device__ __forceinline__ SeqSpan seq_span(const BatchArg& b, int s) {
  SeqSpan x;
  if (b.cu != nullptr) {
    const int end = min(max(b.cu[s + 1], 0), b.n_rows);
    x.first = min(max(b.cu[s], 0), b.n_rows);
    x.n = min(max(end - x.first, 0), b.max_new);
  } else {
    x.first = s * b.max_new;
    x.n = b.max_new;
  }
  x.len = b.len != nullptr ? min(max(b.len[s], 0), b.max_len) : x.n;
  return x;
}

// Sequence of row i, by all lanes of a wave: the number of sequences that end at or before it (those without rows among
// them).  n_seq: behind the last sequence.  All prefix sums are requested at once, so the search costs one trip to memory.
__device__ __forceinline__ int seq_of_row(const BatchArg& b, int i, int lane) {
  if (b.cu == nullptr) return i / b.max_new;
  int n = 0;
  for (int s = 0; s < b.n_seq; s += 64) n += __popcll(__ballot(s + lane < b.n_seq && b.cu[min(s + lane, b.n_seq - 1) + 1] <= i));
  return n;
}

struct AppendLaunch {
  int dtype, d, hq, hkv, rot, interleaved;
  BatchArg b;
  RowsArg k_new, v_new, q, q_out;  // hq = 0: no queries
  const float* inv_freq;           // null: nothing is rotated
  const int32_t* positions;
  char* k;
  char* v;
};
hipError_t launch_paged_append(const AppendLaunch& a, hipStream_t s);

// Attention of the rows of a batch over prompts (k and v as rows) or over pages.
//
// How a batch becomes workgroups.  The rows of a sequence that read one KV head are its tokens' query heads of that group,
// token by token (row t G + g), cut into tiles; the keys that a tile sees are cut into chunks of `chunk` keys, whose partial
// results a second kernel joins.  A work item is (sequence, tile, chunk), a workgroup one item of one KV head.  The grid has
// room for every batch within the host's bounds; which item a workgroup takes, and how long a chunk is, every wave finds from
// the lengths (Items): the keys of all tiles are shared out over as many workgroups as are wanted, so that a
// long sequence among short ones does not hold up the batch.
struct PagedAttnLaunch {
  int dtype, d, hq, hkv, paged;
  BatchArg b;
  RowsArg q, out;
  RowsArg k, v;  // pages: hs = bytes of one head's rows of a page, rs = bytes of a row
  float* lse;    // may be null
  float scale;
  int target_log2, ragged_log2;  // workgroups to share the keys out over, and where sequences differ in length
  int min_chunk;          // keys are shared out in chunks of min_chunk at least (wide tiles: twice that), rounded up to 128
  int max_chunks;         // 1: no sequence's keys are cut
  // partial results of the tiles whose keys are cut, in slots of 32 rows (of tile_rows, where no tile has more)
  int max_slots, tile_rows;
  float* part_o;          // [max_slots][hkv][tile_rows][d], normalised
  float* part_lse;        // [max_slots][hkv][tile_rows], in units of log 2
};
hipError_t launch_paged_attn(const PagedAttnLaunch& a, hipStream_t s);

}  // namespace samkv
