// C ABI of the rotary positions: argument checks and launch plan.  See
// include/ssba_rope.h for the contract.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "ssba_common.h"
#include "ssba_rope_common.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

ssba_status check_rope(const ssba_rope* r) {
  if (!r) return SSBA_ERR_ARG;
  if (r->head_dim != 64 && r->head_dim != 128) return SSBA_ERR_UNSUPPORTED;
  if (r->pairs != SSBA_ROPE_ADJACENT && r->pairs != SSBA_ROPE_HALVES) return SSBA_ERR_ARG;
  if (r->axes < 1 || r->axes > 4) return SSBA_ERR_UNSUPPORTED;
  if (!r->axis || !r->freq) return SSBA_ERR_ARG;
  for (int j = 0; j < r->head_dim / 2; ++j) {
    if (r->axis[j] < -1 || r->axis[j] >= r->axes) return SSBA_ERR_ARG;
    if (!std::isfinite(r->freq[j])) return SSBA_ERR_ARG;
    if (std::fabs(r->freq[j]) > 1048576.0) return SSBA_ERR_UNSUPPORTED;
  }
  return SSBA_OK;
}

// Element strides of a [batch][heads][rows][D] tensor; all 0: contiguous.
// `out`: rows that are written must not overlap.
ssba_status strides_of(int dtype, int64_t batch, int64_t heads, int64_t rows, int d, bool out, int64_t* sb, int64_t* sh,
                       int64_t* st) {
  if (*sb == 0 && *sh == 0 && *st == 0) {
    *st = d;
    *sh = rows * d;
    *sb = heads * rows * d;
  }
  if (*sb < 0 || *sh < 0 || *st < 0) return SSBA_ERR_SHAPE;
  if (rows > 0 && ((rows > 1 && *st < d) || (heads > 1 && *sh < d) || (out && batch > 1 && *sb < d))) return SSBA_ERR_SHAPE;
  if (dtype == SSBA_DT_BF16 && ((*sb | *sh | *st) & 7)) return SSBA_ERR_UNSUPPORTED;
  if ((double)batch * *sb + (double)heads * *sh + (double)rows * *st > 2.0e18) return SSBA_ERR_SHAPE;
  return SSBA_OK;
}

}  // namespace

extern "C" ssba_status ssba_rope_rotate(const ssba_rope* r, int32_t dtype, int32_t inverse, int32_t batch, int32_t rows,
                                        const int32_t* pos, int64_t pos_stride_b, int64_t pos_stride_t, int32_t n,
                                        const ssba_rope_tensor* tensors, void* hip_stream) {
  ssba_status st = check_rope(r);
  if (st != SSBA_OK) return st;
  if (dtype != SSBA_DT_BF16 && dtype != SSBA_DT_F32) return SSBA_ERR_ARG;
  if ((inverse != 0 && inverse != 1) || n < 1 || n > 2 || !tensors) return SSBA_ERR_ARG;
  if (batch < 0 || rows < 0 || pos_stride_b < 0 || pos_stride_t < 0) return SSBA_ERR_SHAPE;
  if ((double)batch * pos_stride_b + (double)rows * pos_stride_t > 2.0e18) return SSBA_ERR_SHAPE;
  ssba::TurnArgs a;
  std::memset(&a, 0, sizeof(a));
  const size_t al = dtype == SSBA_DT_BF16 ? 16 : 4;
  for (int i = 0; i < n; ++i) {
    const ssba_rope_tensor& t = tensors[i];
    if (t.heads < 1) return SSBA_ERR_SHAPE;
    if (t.heads > 65536) return SSBA_ERR_UNSUPPORTED;
    a.heads[i] = t.heads;
    a.x_sb[i] = t.x_stride_b;
    a.x_sh[i] = t.x_stride_h;
    a.x_st[i] = t.x_stride_t;
    a.y_sb[i] = t.y_stride_b;
    a.y_sh[i] = t.y_stride_h;
    a.y_st[i] = t.y_stride_t;
    if ((st = strides_of(dtype, batch, t.heads, rows, r->head_dim, false, &a.x_sb[i], &a.x_sh[i], &a.x_st[i])) != SSBA_OK ||
        (st = strides_of(dtype, batch, t.heads, rows, r->head_dim, true, &a.y_sb[i], &a.y_sh[i], &a.y_st[i])) != SSBA_OK)
      return st;
    if (batch > 0 && rows > 0 && (!t.x || !t.y)) return SSBA_ERR_ARG;
    if (!aligned(t.x, al) || !aligned(t.y, al)) return SSBA_ERR_ARG;
    if (t.x == t.y && (a.x_sb[i] != a.y_sb[i] || a.x_sh[i] != a.y_sh[i] || a.x_st[i] != a.y_st[i])) return SSBA_ERR_ARG;
    a.x[i] = static_cast<const char*>(t.x);
    a.y[i] = static_cast<char*>(t.y);
  }
  if (batch == 0 || rows == 0) return SSBA_OK;
  if (!pos || !aligned(pos, 4)) return SSBA_ERR_ARG;
  a.pos = pos;
  a.p_sb = pos_stride_b;
  a.p_st = pos_stride_t;
  a.rows = rows;
  a.tokens = (int64_t)batch * rows;
  a.inverse = inverse;
  const double quarter = 0.63661977236758134308;   // 2 / pi
  for (int j = 0; j < r->head_dim / 2; ++j) {
    a.axis[j] = (int8_t)r->axis[j];
    a.freq[j] = r->freq[j] * quarter;
  }
  // The heads of a few tokens are shared by several workgroups, of 4 heads or more each.
  const int64_t tiles = (a.tokens + ssba::kRopeRows - 1) / ssba::kRopeRows;
  const int all = a.heads[0] + a.heads[1];
  a.head_parts = (int)std::max<int64_t>(1, std::min<int64_t>((all + 3) / 4, 256 / tiles));
  if (tiles * a.head_parts > ssba::kMaxGroups256) return SSBA_ERR_UNSUPPORTED;
  return ssba::launch_rope_turn(a, r->head_dim, dtype, r->pairs, static_cast<hipStream_t>(hip_stream)) == hipSuccess
             ? SSBA_OK
             : SSBA_ERR_HIP;
}
