// Internal declarations of the rotary positions (include/ssba_rope.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssba_rope.h"

namespace ssba {

struct TurnArgs {
  const char* x[2];
  char* y[2];
  int64_t x_sb[2], x_sh[2], x_st[2];   // elements
  int64_t y_sb[2], y_sh[2], y_st[2];
  int heads[2];
  const int32_t* pos;
  int64_t p_sb, p_st;
  int rows;
  int64_t tokens;      // batch * rows
  int head_parts;      // workgroups that share a tile's heads
  int inverse;
  double freq[64];     // quarter turns a position
  int8_t axis[64];     // -1: the pair stays
};

constexpr int kRopeRows = 4;   // tokens of a workgroup

hipError_t launch_rope_turn(const TurnArgs& a, int head_dim, int dtype, int pairs, hipStream_t s);

}  // namespace ssba
