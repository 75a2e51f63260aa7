// Internal declarations of the windowed attention (include/ssba_window.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssba_window.h"

namespace ssba {

struct Strides {
  int64_t b, h, t;   // elements
};

constexpr int kWindowRows = 128;   // rows of a workgroup: 32 a wave

struct WindowArgs {
  const void* q;
  const void* k;
  const void* v;
  void* o;             // backward: read
  float* lse;
  const void* dout;    // backward
  void* dq;
  void* dk;
  void* dv;
  float* lse2;         // backward scratch: lse in log2 units, -delta [batch][heads][seq]
  float* ndelta;
  float* part;         // parts of dk and dv [unit][sink tile and chunk slot, then slot][share][2][128][D]
  Strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  const int32_t* cu;
  int batch, seq, heads, kv_heads, group, window, sinks, seqs;
  float scale, scale_log2;
  int slots;           // tiles of kWindowRows rows of a (batch, head): packed ones with unused slots between
  int spread;          // order of the workgroups, see place()
  int sink_tiles;      // tiles of kWindowRows keys that hold sinks
  int chunk;           // queries of a chunk of a sink tile
  int chunk_slots;     // of a (batch, head): 0: no tile is cut
  int head_parts;      // key side: workgroups that share the heads of a group,
  int query_parts;     // and the queries of a tile or chunk
};

// Whether a launch of `groups` workgroups takes 8 waves, in two groups that
// share the tiles: where the chip has room for them (one workgroup a CU) and
// there are tiles to share.  One group against two, forward and backward, in us:
// 1024 rows, 16 heads on 4, window 1024: bf16 D 64 18.0 to 15.6 and 56.5 to 48.9,
// D 128 25.9 to 22.5 and 83.3 to 80.5, fp32 D 64 55 to 41 and 164 to 137.  But
// 384 tiles of bf16 D 64 16.9 to 21.9 and 69 to 74, 100 rows of window 64 6.6 to
// 7.1 and 16.1 to 18.0.  fp32 D 64 on the key side up to 1024 (4096 rows, 16 heads
// on 4, window 1000: backward 428 to 400; 12 heads, window 300: 174 to 151).  fp32
// D 128 needs the registers of two waves for one.
inline bool share_tiles(const WindowArgs& a, unsigned groups, unsigned most = 256) {
  return groups <= most && (int64_t)a.window + a.sinks >= 256;
}

hipError_t launch_window_forward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s);
hipError_t launch_window_backward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s);

}  // namespace ssba
