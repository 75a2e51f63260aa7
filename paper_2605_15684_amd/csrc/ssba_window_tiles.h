// What the windowed attention's forward and backward share: which rows a
// workgroup has, tiles of rows in the LDS, and the two kinds of product.
//
// A tile is 32 or 64 rows, in halves of 32 that buffer_load ... lds fills.  Products are 32 x 32 by
// v_mfma_f32_32x32x16_bf16 or v_mfma_f32_32x32x2_f32, whose result gives lane l
// column l % 32 and rows 8 (e / 4) + 4 (l / 32) + e % 4, e = 0 .. 15:
//   rows_product   (tile rows) x (the wave's 32 rows, in registers)
//   cols_product   (tile columns)^T x (such a result, in registers)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ssba_tiles.h"
#include "ssba_window_common.h"

namespace ssba {

typedef float floatx4 __attribute__((ext_vector_type(4)));

enum WKind {
  kBf16,
  kF32,      // fp32 as it is, products by v_mfma_f32_32x32x2_f32
  kF32Split  // each value as three bf16 terms that make it up exactly, in three planes; products by
             // v_mfma_f32_32x32x16_bf16, of the six pairs of terms that reach 2^-24 of the product (the others are at
             // most 2^-24 of it): 192 cycles for 16 channels instead of 512.  An infinity becomes NaN.
};

template <int D_, int KIND, int NB_ = KIND == kBf16 ? 2 : 1>
struct WTile {
  static constexpr int D = D_;
  static constexpr bool F32 = KIND != kBf16, NATIVE = KIND == kF32, SPLIT = KIND == kF32Split;
  static constexpr int SIZE = F32 ? 4 : 2;      // bytes of a value in memory
  static constexpr int ROWB = D * (NATIVE ? 4 : 2);   // bytes of a row in the LDS
  static constexpr int CPR = ROWB / 16;         // 16-byte chunks of a row
  static constexpr int NB = NB_;                // halves of a tile
  static constexpr int PL = SPLIT ? 3 : 1;      // planes
  static constexpr int ROWS = 32 * NB;
  static constexpr int HALF = 32 * ROWB;
  static constexpr int TILE = PL * NB * HALF;   // 8 to 24 KB
  // Registers are short and two waves a SIMD few: reads and products are put in order by hand.
  static constexpr bool ORDERED = D == 128 && !F32;
  static constexpr int KPI = 1024 / ROWB;       // rows of a copy instruction
  static constexpr int NIW = TILE / 4096;       // copy instructions of each of 4 waves
  static constexpr int NU = D / 64;             // SPLIT: eights of a thread in a tile
  static constexpr int NKS = NATIVE ? D / 8 : D / 16;   // 16-byte operands of a lane in a row
  static constexpr int NDB = D / 32;
  static_assert(!SPLIT || NB == 1, "planes follow each other");
};

template <class T>
__device__ __forceinline__ int wswz(int k, int c) {
  if constexpr (T::NATIVE)
    return c ^ (k & 7);
  else
    return swz<T::D>(k, c);
}

// a and b as N bf16 terms each, every one the rounding of what the ones before
// leave: of 3 (fp32 made up exactly) the second is at most 2^-8, the third 2^-16
// of the value.
template <int N>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = pack2(a, b);
    a -= __uint_as_float(t[i] << 16);
    b -= __uint_as_float(t[i] & 0xFFFF0000u);
  }
}

// The rows of a workgroup: of sequence (batch b or packed), head h.
struct WPlace {
  int b, h, kvh, g;
  int begin, len;   // the sequence's rows
  int r0;           // first row of the workgroup in the sequence
};

// The sequence whose slots include slot x, where sequence s has the slots from
// cu[s] / rows + s on (its tiles need no more of them than the next one's
// first).  One wave, every lane gets the result.
__device__ __forceinline__ int seq_of_slot(const int32_t* cu, int seqs, int seq, int rows, int x, int lane) {
  int lo = 0, n = seqs;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int s = lo + lane * step;
    const bool in = lane * step < n && min(max(cu[min(s, seqs - 1)], 0), seq) / rows + s <= x;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(in));   // cu does not decrease: the first c lanes
    lo += max(c - 1, 0) * step;
    n = min(step, seqs - lo);
  }
  return lo;
}

__device__ __forceinline__ void seq_rows(const WindowArgs& a, int s, int* begin, int* len) {
  *begin = min(max(a.cu[s], 0), a.seq);
  *len = max(min(a.cu[s + 1], a.seq), *begin) - *begin;
}

// Workgroup `id` of `n` -> position in the launch's order.  The workgroups of
// one XCD (id mod 8) are consecutive, so that the heads of a group and
// neighbouring tiles read their rows from one L2.
__device__ __forceinline__ unsigned xcd_order(unsigned id, unsigned n) {
  const unsigned per = n / 8, rest = n % 8, x = id % 8;
  return x * per + min(x, rest) + id / 8;
}

// Slot of a (batch, head) -> rows.  False: none.
__device__ __forceinline__ bool place_slot(const WindowArgs& a, int slot, int lane, WPlace* p) {
  if (a.cu) {
    const int s = seq_of_slot(a.cu, a.seqs, a.seq, kWindowRows, slot, lane);
    seq_rows(a, s, &p->begin, &p->len);
    p->r0 = (slot - (p->begin / kWindowRows + s)) * kWindowRows;
  } else {
    p->begin = 0;
    p->len = a.seq;
    p->r0 = slot * kWindowRows;
  }
  return p->r0 >= 0 && p->r0 < p->len;
}

// The workgroup's rows and head, of launches with a workgroup for each slot and
// query head.
__device__ __forceinline__ bool place_query(const WindowArgs& a, int lane, WPlace* p) {
  const unsigned units = (unsigned)a.batch * a.kv_heads;
  unsigned unit, slot;
  if (a.spread) {   // tiles of every head in turn, last ones (long ones) first
    unsigned id = blockIdx.x;
    unit = id % units;
    id /= units;
    p->g = id % a.group;
    slot = a.slots - 1 - id / a.group;
  } else {
    unsigned id = xcd_order(blockIdx.x, gridDim.x);
    p->g = id % a.group;
    id /= a.group;
    slot = a.slots - 1 - id % a.slots;
    unit = id / a.slots;
  }
  p->b = unit / a.kv_heads;
  p->kvh = unit % a.kv_heads;
  p->h = p->kvh * a.group + p->g;
  return place_slot(a, slot, lane, p);
}

// 1 KB from the `bytes` behind p, zeros for what is past them.
__device__ __forceinline__ void copy_kb(const char* p, unsigned bytes, unsigned off, char* dst) {
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, (int)bytes, kRawBufferFlags);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 16, off, 0, 0, 0);
}

// 16 bytes from the `bytes` behind p, zeros for what is past them.
__device__ __forceinline__ floatx4 load_bounded(const char* p, unsigned bytes, unsigned off) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0, (int)bytes, kRawBufferFlags);
  const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0);
  return __builtin_bit_cast(floatx4, x);
}

// This wave's copy of its part of a tile: rows row0 .. of a (b, h) slice, rows
// from `end` on become 0.  issue() begins it; land() behind the work that hides
// it, then a wait for vector memory and a barrier, end it.  SPLIT: the values
// pass through registers, where they are split.
template <class T>
struct WCopy {
  const char* base;   // row 0
  unsigned rowb;      // bytes from row to row
  unsigned off[T::SPLIT ? 1 : T::NIW];
  floatx4 held[T::SPLIT ? 2 * T::NU : 1];
  __device__ __forceinline__ void init(const void* p, int64_t elem, int64_t st, int wave, int lane) {
    base = static_cast<const char*>(p) + elem * T::SIZE;
    rowb = (unsigned)st * T::SIZE;
    if constexpr (T::SPLIT) {
      const int u = 64 * wave + lane;
      off[0] = (unsigned)(u / (T::D / 8)) * rowb + 32u * (unsigned)(u % (T::D / 8));
    } else {
#pragma unroll
      for (int m = 0; m < T::NIW; ++m) {
        const int row = T::KPI * (T::NIW * wave + m) + lane / T::CPR;
        off[m] = (unsigned)row * rowb + 16u * (unsigned)wswz<T>(row & 31, lane % T::CPR);
      }
    }
  }
  __device__ __forceinline__ void issue(int row0, int end, char* dst, int wave) {
    const int left = min(end - row0, T::ROWS);
    const unsigned bytes = left > 0 ? (unsigned)(left - 1) * rowb + T::D * T::SIZE : 0u;
    const char* from = base + (int64_t)row0 * rowb;
    if constexpr (T::SPLIT) {
#pragma unroll
      for (int i = 0; i < T::NU; ++i) {
        const unsigned at = off[0] + (unsigned)(i * (2048 / T::D)) * rowb;   // 256 eights are 2048 / D rows
        held[2 * i] = load_bounded(from, bytes, at);
        held[2 * i + 1] = load_bounded(from, bytes, at + 16);
      }
    } else {
#pragma unroll
      for (int m = 0; m < T::NIW; ++m) copy_kb(from, bytes, off[m], dst + 1024 * (T::NIW * wave + m));
    }
  }
  __device__ __forceinline__ void land(char* dst, int wave, int lane) const {
    if constexpr (T::SPLIT) {
#pragma unroll
      for (int i = 0; i < T::NU; ++i) {
        const int u = 64 * wave + lane + 256 * i, row = u / (T::D / 8), c = u % (T::D / 8);
        uint32_t w[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t x[3];
          split2(held[2 * i + e / 2][2 * (e & 1)], held[2 * i + e / 2][2 * (e & 1) + 1], x);
#pragma unroll
          for (int t = 0; t < 3; ++t) w[t][e] = x[t];
        }
        char* to = dst + row * T::ROWB + 16 * wswz<T>(row, c);
#pragma unroll
        for (int t = 0; t < 3; ++t)
          *reinterpret_cast<uint4*>(to + t * T::HALF) = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
      }
    }
  }
};

// 16 bytes of a lane's row: the operands of rows_product, the lane's half of the
// row (lane / 32).
template <class T>
struct WRow {
  floatx4 f[T::PL][T::NKS];
  __device__ __forceinline__ void load(const char* row, int hw) {
#pragma unroll
    for (int ks = 0; ks < T::NKS; ++ks) {
      if constexpr (T::SPLIT) {
        uint32_t w[3][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const floatx4 x = *reinterpret_cast<const floatx4*>(row + 64 * ks + 32 * hw + 16 * h);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t y[3];
            split2(x[2 * e], x[2 * e + 1], y);
#pragma unroll
            for (int t = 0; t < 3; ++t) w[t][2 * h + e] = y[t];
          }
        }
#pragma unroll
        for (int t = 0; t < 3; ++t)
          f[t][ks] = __builtin_bit_cast(floatx4, make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]));
      } else {
        f[0][ks] = *reinterpret_cast<const floatx4*>(row + 32 * ks + 16 * hw);
      }
    }
  }
};

// One such operand as a copy in the LDS in the order of its use: 1 KB each.
template <class T>
struct WRowLds {
  const char* at;   // the wave's, lane's 16 bytes of the first
};
template <class T>
__device__ __forceinline__ floatx4 operand(const WRow<T>& r, int ks, int plane) {
  return r.f[plane][ks];
}
template <class T>
__device__ __forceinline__ floatx4 operand(const WRowLds<T>& r, int ks, int) {
  return *reinterpret_cast<const floatx4*>(r.at + 1024 * ks);
}

// Where a lane's operands lie in a half tile: all of one kind differ by
// exclusive ors and sums of constants.
template <class T>
struct WLane {
  int row, col;
  __device__ __forceinline__ explicit WLane(int lane) {
    const int l32 = lane & 31, hw = lane >> 5;
    row = l32 * T::ROWB + 16 * wswz<T>(l32, hw);
    if constexpr (T::NATIVE) {
      col = 4 * hw * T::ROWB + 16 * wswz<T>(4 * hw, l32 >> 2) + 4 * (l32 & 3);
    } else {
      // As tr_frag: rows 4 hw + li / 4, channels 16 (G & 1) + 4 (li & 3) ..
      const int G = lane >> 4, li = lane & 15, k = 4 * hw + (li >> 2), ch = 16 * (G & 1) + 4 * (li & 3);
      col = k * T::ROWB + 16 * wswz<T>(k, ch >> 3) + 2 * (ch & 7);
    }
  }
  // Forgotten by the compiler, which would otherwise keep every address in a
  // register and spill.
  __device__ __forceinline__ void forget() {
    if constexpr (T::ORDERED) asm volatile("" : "+v"(row), "+v"(col));
  }
};

// Row l % 32, the 16-byte chunk 2 ks + l / 32.
template <class T>
__device__ __forceinline__ floatx4 row_operand(const char* half, const WLane<T>& l, int ks) {
  return *reinterpret_cast<const floatx4*>(half + (l.row ^ (32 * ks)));
}

// bf16: channels 32 db .. of rows 16 ks + 8 (e / 4) + 4 (l / 32) + e % 4.
template <class T>
__device__ __forceinline__ bf16x8 col_operand(const char* half, const WLane<T>& l, int ks, int db) {
  s16x4 x[2];
#pragma unroll
  for (int rr = 0; rr < 2; ++rr)
    x[rr] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4*)(half + (l.col ^ (64 * db + 32 * rr)) + (8 * rr + 16 * ks) * T::ROWB));
  return __builtin_bit_cast(bf16x8, s16x8{x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]});
}

template <class T>
__device__ __forceinline__ void multiply(floatx16& acc, floatx4 x, floatx4 y) {
  if constexpr (T::NATIVE) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
  } else {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
  }
}

// acc += operand ks of the half's rows times that of b: small pairs of terms first,
// and of these the half's largest term first, or b's (B_FIRST): with it the two
// change places and the sum stays the same to the bit.
template <class T, bool B_FIRST, class Row>
__device__ __forceinline__ void row_step(floatx16& acc, const char* half, const Row& b, const WLane<T>& l, int ks) {
  floatx4 x[T::PL];
#pragma unroll
  for (int i = 0; i < T::PL; ++i) {
    const int t = B_FIRST ? T::PL - 1 - i : i;
    x[t] = row_operand<T>(half + t * T::HALF, l, ks);
  }
#pragma unroll
  for (int sum = T::PL - 1; sum >= 0; --sum)
#pragma unroll
    for (int t = 0; t <= sum; ++t)
      multiply<T>(acc, x[B_FIRST ? sum - t : t], operand<T>(b, ks, B_FIRST ? t : sum - t));
}

template <class T>
__device__ __forceinline__ void rows_product(floatx16& acc, const char* half, const WRow<T>& b, const WLane<T>& l) {
#pragma unroll
  for (int ks = 0; ks < T::NKS; ++ks) row_step<T, false>(acc, half, b, l, ks);
}

// Two of them in turn.
template <class T, bool B_FIRST, class Row1, class Row2>
__device__ __forceinline__ void rows_products(floatx16& acc1, const char* half1, const Row1& b1, floatx16& acc2,
                                              const char* half2, const Row2& b2, const WLane<T>& l) {
#pragma unroll
  for (int ks = 0; ks < T::NKS; ++ks) {
    row_step<T, B_FIRST>(acc1, half1, b1, l, ks);
    row_step<T, B_FIRST>(acc2, half2, b2, l, ks);
  }
}

// acc[db] += (channels 32 db .. of the half's rows)^T x, x a 32 x 32 result.
// TERMS: bf16 terms of x, each the rounding of what the ones before leave.
template <class T, int TERMS = 1>
__device__ __forceinline__ void cols_product(floatx16 (&acc)[T::NDB], const char* half, const floatx16& x, const WLane<T>& l) {
  if constexpr (T::NATIVE) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
#pragma unroll
      for (int db = 0; db < T::NDB; ++db) {
        const float w = *reinterpret_cast<const float*>(half + (l.col ^ (16 * (j & 3))) +
                                                        (8 * (j >> 2) + (j & 3)) * T::ROWB + 128 * db);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(w, x[j], acc[db], 0, 0, 0);
      }
  } else if constexpr (T::SPLIT) {
    uint32_t pk[3][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[3];
      split2(x[2 * j], x[2 * j + 1], w);
#pragma unroll
      for (int t = 0; t < 3; ++t) pk[t][j] = w[t];
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < T::NDB; ++db) {
        bf16x8 w[3];
#pragma unroll
        for (int t = 0; t < 3; ++t) w[t] = col_operand<T>(half + t * T::HALF, l, ks, db);
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int t = 0; t <= sum; ++t)
            acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[t], packed_frag(pk[sum - t], ks), acc[db], 0, 0, 0);
      }
  } else {
    uint32_t pk[TERMS][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t w[TERMS];
      split2(x[2 * j], x[2 * j + 1], w);
#pragma unroll
      for (int t = 0; t < TERMS; ++t) pk[t][j] = w[t];
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int db = 0; db < T::NDB; ++db) {
        const bf16x8 w = col_operand<T>(half, l, ks, db);
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t)
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, packed_frag(pk[t], ks), acc[db], 0, 0, 0);
      }
  }
}

// The same where rows that a column does not see must not reach it whatever
// they hold (0 times NaN): one row after another.  `seen`: a bit for each row
// that this lane's column sees.  `room`: 4 KB of LDS of the wave.
template <class T>
__device__ __forceinline__ void cols_product_seen(floatx16 (&acc)[T::NDB], const char* half, const floatx16& x,
                                                            float* room, int lane, uint32_t seen) {
  const int l32 = lane & 31, hw = lane >> 5;
#pragma unroll
  for (int j = 0; j < 16; ++j) room[j * 64 + lane] = x[j];
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int db = 0; db < T::NDB; ++db)
#pragma unroll 1
    for (int row = 0; row < 32; ++row) {
      const int j = 4 * (row >> 3) + (row & 3), from = (row >> 2) & 1;
      const float w = room[j * 64 + l32 + 32 * from];
      const bool in = (seen >> row) & 1;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int ch = 32 * db + 8 * (e >> 2) + 4 * hw + (e & 3), at = ch * T::SIZE;
        const char* p = half + row * T::ROWB + 16 * wswz<T>(row, at >> 4) + (at & 15);
        float y;
        if constexpr (T::NATIVE)
          y = *reinterpret_cast<const float*>(p);
        else
          y = __uint_as_float((uint32_t)*reinterpret_cast<const u16*>(p) << 16);
        acc[db][e] = in ? __builtin_fmaf(w, y, acc[db][e]) : acc[db][e];
      }
    }
  __builtin_amdgcn_wave_barrier();
}

// A result as rows of the lane's column: 4 consecutive channels at a time, of
// the first N blocks of acc.
template <class T, int N = T::NDB>
__device__ __forceinline__ void store_cols(char* row, const floatx16 (&acc)[T::NDB], float f, int hw) {
#pragma unroll
  for (int db = 0; db < N; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x[4] = {acc[db][4 * j] * f, acc[db][4 * j + 1] * f, acc[db][4 * j + 2] * f, acc[db][4 * j + 3] * f};
      char* p = row + (32 * db + 8 * j + 4 * hw) * T::SIZE;
      if constexpr (T::F32)
        *reinterpret_cast<floatx4*>(p) = floatx4{x[0], x[1], x[2], x[3]};
      else
        *reinterpret_cast<uint2*>(p) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
    }
}

// The sums of two groups of four waves that had the same rows or keys: group 0
// has the first half of the channel blocks of both then, group 1 the second, in
// acc[0 .. NDB / 2 - 1].  A quarter of the passed values goes through each buffer:
// NDB / 2 * 8 KB of them.
template <int NDB>
__device__ __forceinline__ void join_groups(floatx16 (&acc)[NDB], int group, int thread, char* b0, char* b1, char* b2, char* b3) {
  float* const room[4] = {reinterpret_cast<float*>(b0), reinterpret_cast<float*>(b1), reinterpret_cast<float*>(b2),
                          reinterpret_cast<float*>(b3)};
  constexpr int H = NDB / 2, PER = 4 * H;   // values of a thread in a buffer
  // Selected by bits: a choice of registers by index would put them into memory.
  const uint32_t second = group ? ~0u : 0u;
  auto pick = [&](float x, float y) {
    return __uint_as_float((__float_as_uint(x) & ~second) | (__float_as_uint(y) & second));
  };
  __syncthreads();
#pragma unroll
  for (int db = 0; db < H; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int n = 16 * db + e;
      room[n / PER][(group * PER + n % PER) * 256 + thread] = pick(acc[db + H][e], acc[db][e]);
      acc[db][e] = pick(acc[db][e], acc[db + H][e]);
    }
  __syncthreads();
#pragma unroll
  for (int db = 0; db < H; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int n = 16 * db + e;
      acc[db][e] += room[n / PER][((1 - group) * PER + n % PER) * 256 + thread];
    }
}

// Some element is not finite.
template <int N>
__device__ __forceinline__ bool not_finite(const floatx16 (&acc)[N]) {
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) t = __builtin_fmaf(acc[i][e], 0.f, t);
  return t != 0.f;   // NaN
}

// The low n bits, n clamped to 0 .. 32.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : ~0u >> (32 - min(n, 32)); }

// Which of the tokens j0 .. j0 + 31 token i sees, a bit each.
__device__ __forceinline__ uint32_t keys_seen(int i, int j0, int window, int sinks) {
  return low_bits(i + 1 - j0) & (~low_bits(i + 1 - window - j0) | low_bits(sinks - j0));
}

// Which of the tokens i0 .. i0 + 31, of q0 .. q1 - 1, see token j.
__device__ __forceinline__ uint32_t queries_seeing(int j, int i0, int q0, int q1, int window, int sinks) {
  const int end = j < sinks ? q1 : min(q1, j + window);
  return low_bits(end - i0) & ~low_bits(max(j, q0) - i0);
}

// Of such bits, all ones or zeros for element e of a 32 x 32 result (its row
// 8 (e / 4) + 4 hw + e % 4); `bits` shifted right by 4 hw.
__device__ __forceinline__ uint32_t bit_of(uint32_t bits, int e) {
  return (uint32_t)((int32_t)(bits << (31 - (8 * (e >> 2) + (e & 3)))) >> 31);
}
__device__ __forceinline__ float keep_if(uint32_t ones, float x) { return __uint_as_float(__float_as_uint(x) & ones); }

}  // namespace ssba
