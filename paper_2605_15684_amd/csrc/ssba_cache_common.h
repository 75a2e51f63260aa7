// Internal declarations of the paged 8-bit key/value cache (include/ssba_cache.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssba_cache.h"

namespace ssba {

// One layer of a cache.
struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* scale;      // [pages][kv_heads][2]
  uint16_t* kmean;   // [pages][kv_heads][D]
  int64_t page_bytes;  // kv_heads * page * D: one page of k or v
  int pages, kv_heads, head_dim;
  int page_log2;
};

struct BatchView {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
  int seqs, max_pages, rows, max_new;
};

// A sequence of the batch as the kernels see it: whatever the arrays hold,
// begin + n <= rows and 0 <= len <= max_pages * page.  The first of the n new
// tokens is at position start: negative where the sequence holds fewer, len
// where it has outgrown its table by all of them.
struct SeqView {
  int begin, n, start, len;
};

__device__ __forceinline__ SeqView seq_view(const BatchView& b, int page_log2, int s) {
  SeqView v;
  v.begin = min(max(b.cu[s], 0), b.rows);
  v.n = max(min(b.cu[s + 1], b.rows), v.begin) - v.begin;
  const int all = max(b.lens[s], 0);
  v.len = min(all, b.max_pages << page_log2);
  v.start = min(all - v.n, v.len);
  return v;
}

// The sequence of packed row r and its view; false if the row is no
// sequence's new token.  One wave, every lane gets the result.  The sequence
// is the number of ends cu[1..seqs] that are <= r (cu does not decrease); a
// lane holds one end and the length of the sequence that begins behind the
// last one, so that nothing is loaded after the search.
__device__ __forceinline__ bool seq_of_row(const BatchView& b, int page_log2, int r, int lane, int* seq, SeqView* v) {
  int begin = b.cu[0];
  for (int j0 = 1; j0 <= b.seqs; j0 += 64) {
    const int j = j0 + lane;
    const bool in = j <= b.seqs;
    const int end = in ? b.cu[j] : 0, len = in ? b.lens[j - 1] : 0;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(in && end <= r));
    if (c > 0) begin = __builtin_amdgcn_readlane(end, c - 1);
    if (c < 64) {
      *seq = j0 - 1 + c;
      if (*seq >= b.seqs) return false;
      v->begin = min(max(begin, 0), b.rows);
      v->n = max(min(__builtin_amdgcn_readlane(end, c), b.rows), v->begin) - v->begin;
      const int all = max(__builtin_amdgcn_readlane(len, c), 0);
      v->len = min(all, b.max_pages << page_log2);
      v->start = min(all - v->n, v->len);
      return r >= v->begin && r - v->begin < v->n;
    }
  }
  return false;
}

struct AppendArgs {
  CacheView c;
  BatchView b;
  const void* k;
  const void* v;
  int64_t st, sh;
  int slots;   // pages a sequence can touch
};

struct SelectArgs {
  CacheView c;
  BatchView b;
  const void* q;
  int64_t st, sh;
  int32_t* lists;
  uint64_t* keys;   // [rows][kv_heads][max_pages] ranking keys of the scored pages
  int group, causal, keep, first, last;
  int tiles;        // tiles of 16 tokens of a sequence
};
constexpr int kSelectPages = 64;     // pages a workgroup scores at a time
constexpr int kSelectInLds = 1152;   // pages whose scores of 16 tokens the LDS holds (144 of its 160 KB)

// What the selection launches (ssba_cache_api.cpp decides).
enum SelectKind { kSelectRow, kSelectTile, kSelectRowLong, kSelectTileLong };
struct SelectPlan {
  SelectKind kind;
  int chunks;       // long kinds: workgroups that share a row's (a tile's) pages
  bool scored;      // long kinds: some row may have pages to score
};

struct AttendArgs {
  CacheView c;
  BatchView b;
  const void* q;
  void* o;
  int64_t q_st, q_sh, o_st, o_sh;
  const int32_t* lists;   // [rows][kv_heads][1 + keep] or null
  float* part;            // parts of split items: O [item][split][columns][D]
  float* part_ml;         // and their maximum and sum [item][split][columns][2]
  float scale_log2;
  int group, causal, keep;
  int col_tiles;          // column tiles of an item
  int splits;             // workgroups that share an item's keys
  // What follows is read by the kinds of its name only.
  int window, sinks;      // kAttendWindow; window <= 2^30
  const int32_t* first;   // kAttendShared: [groups + 1] first sequence of each group
  const int32_t* shared;  // [groups] pages of its prefix
  int groups, shared_cols;   // shared_cols: most columns of a group
  int tiles;              // tiles of 16 columns of an item
  float* prefix_part;     // part and part_ml of the prefixes
  float* prefix_ml;
  int prefix_cols, prefix_col_tiles, prefix_splits;   // of the prefixes: columns of an item, most column tiles, splits
  int prefix_slots;       // column tiles of all groups where they are packed, 0: prefix_col_tiles for each
};

// What the attention launch does (ssba_cache_api.cpp decides).
enum AttendKind {
  kAttendSeq,    // items: (sequence, kv head, column tile)
  kAttendRow,    // lists; items: (row, kv head, column tile), the waves of a workgroup share the keys
  kAttendRows,   // lists; a wave per such item
  kAttendWindow, // as kAttendSeq, keys of the sinks and the window
  kAttendShared, // as kAttendSeq for what is behind the prefixes; items of these: (group, kv head, column tile), or
                 // (slot, kv head) where the groups' column tiles are packed
};
struct AttendPlan {
  AttendKind kind;
  int tiles;              // tiles of 16 columns of an item
  int threads;
  int col_tiles, splits;
  int64_t items;          // workgroups without the splits
  int prefix_tiles, prefix_threads, prefix_col_tiles, prefix_splits, prefix_slots;   // kAttendShared: the same of the prefixes
  int64_t prefix_items;
};

hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t s);
hipError_t launch_cache_select(const SelectArgs& a, const SelectPlan& p, int dtype, hipStream_t s);
hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s);

struct PagesArgs {
  int rows, max_pages, pages, page_log2;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int32_t* info;
  int32_t* scratch;
  const int32_t* src;
  const int32_t* dst;
  int32_t* table_out;
  int32_t* refs_out;
  int n;
};
// A whole cache for page copies: per page and layer the bytes of each array.
struct CopyArgs {
  const char* from[4];
  char* to[4];
  int64_t bytes[4];          // per page
  int64_t from_layer[4], to_layer[4];   // bytes per layer
  int layers, from_pages, to_pages;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* count;      // pairs (null: n)
  int n;
  // A compaction's page table: table_out[e] = map[table[e]] (map null: none).
  const int32_t* map;
  const int32_t* table;
  int32_t* table_out;
  int64_t entries;
};

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_release(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_copy(const CopyArgs& a, hipStream_t s);

}  // namespace ssba
