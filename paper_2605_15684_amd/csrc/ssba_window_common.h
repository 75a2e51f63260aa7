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
  float* part;         // parts of dk and dv [unit][sink tile and chunk slot, then slot][share of the heads][2][128][D]
  Strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  const int32_t* cu;
  int batch, seq, heads, kv_heads, group, window, sinks, seqs;
  float scale, scale_log2;
  int slots;           // tiles of kWindowRows rows of a (batch, head): packed ones with unused slots between
  int spread;          // order of the workgroups, see place()
  int sink_tiles;      // tiles of kWindowRows keys that hold sinks
  int chunk;           // queries of a chunk of a sink tile
  int chunk_slots;     // of a (batch, head): 0: no tile is cut
  int head_parts;      // workgroups that share the heads of a group on the key side
};

hipError_t launch_window_forward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s);
hipError_t launch_window_backward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s);

}  // namespace ssba
