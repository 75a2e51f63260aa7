// Tiles of rows in the LDS and their operands of v_mfma_f32_32x32x16_bf16, for
// the kernels that keep bf16 rows in half tiles of 32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ssba {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kWaitVm0 = 0x0F70;          // s_waitcnt: every vector memory operation done
constexpr int kRawBufferFlags = 0x00020000;
constexpr float kLog2e = 1.4426950408889634f;
// sched_group_barrier classes.
constexpr int kMfma = 0x8, kDsRead = 0x100;

template <int D>
struct BShape {
  static constexpr int CPR = D / 8;            // 16-byte chunks per row
  static constexpr int ROWB = 2 * D;           // bytes per row
  static constexpr int KPI = 1024 / ROWB;      // rows per copy instruction
  static constexpr int NI = 32 / KPI;          // copy instructions per 32-row half
  static constexpr int NIW = NI / 2;           // ... per wave (two waves share a half)
  static constexpr int HALF = 32 * ROWB;       // bytes of a half tile
  static constexpr int NKS = D / 16;           // 16-channel steps of a row product
  static constexpr int NDB = D / 32;           // 32-channel output tiles
};

// Physical 16-byte chunk of logical chunk c in row k (0..31) of a half tile.
// Chosen (by exhaustive search over XOR maps of the row bits) so that both the
// 16-byte row reads of 32 rows at one chunk and the transposed 8-byte reads of
// four rows x four channel quads hit distinct banks.
template <int D>
__device__ __forceinline__ int swz(int k, int c) {
  if constexpr (D == 64)
    return c ^ ((4 * ((k >> 1) & 1)) ^ ((k >> 2) & 1) ^ (2 * ((k >> 3) & 1)));
  else
    return c ^ ((4 * (k & 1)) ^ (8 * ((k >> 1) & 1)) ^ ((k >> 2) & 1) ^ (2 * ((k >> 3) & 1)));
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{lo, hi}, bf16x2));
}

// Row operand of a 32x32x16 product from a half tile: row l % 32, logical
// chunk 2 ks + l / 32 (eight consecutive channels).
template <int D>
__device__ __forceinline__ bf16x8 row_frag(const char* half, int lane, int ks) {
  const int k = lane & 31, c = 2 * ks + (lane >> 5);
  return *reinterpret_cast<const bf16x8*>(half + k * BShape<D>::ROWB + 16 * swz<D>(k, c));
}

// Transposed operand (channels x rows) of a 32x32x16 product from a half
// tile: 32 channels 32 db + (lane % 32) ... as the hardware transposing read
// lays them out, over rows 16 ks + 8 (e / 4) + 4 (lane / 32) + e % 4.
template <int D>
__device__ __forceinline__ s16x8 tr_frag(const char* half, int lane, int ks, int db) {
  const int G = lane >> 4, li = lane & 15, hw = lane >> 5;
  const int ch = 32 * db + 16 * (G & 1) + 4 * (li & 3);
  const int c = ch >> 3, off = 2 * (ch & 7);
  s16x4 x[2];
#pragma unroll
  for (int rr = 0; rr < 2; ++rr) {
    const int k = 16 * ks + 8 * rr + 4 * hw + (li >> 2);
    x[rr] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4*)(half + k * BShape<D>::ROWB + 16 * swz<D>(k, c) + off));
  }
  return s16x8{x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
}

// B operand from registers: P^T / dS^T rows 16 ks + 8 (e / 4) + 4 (lane / 32) + e % 4.
__device__ __forceinline__ bf16x8 packed_frag(const uint32_t (&pk)[8], int ks) {
  return __builtin_bit_cast(bf16x8, make_uint4(pk[4 * ks], pk[4 * ks + 1], pk[4 * ks + 2], pk[4 * ks + 3]));
}

// Sum of v over lanes l and l ^ 32 (the swap returns both halves' values).
__device__ __forceinline__ float swap_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace ssba
