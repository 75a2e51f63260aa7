// Attention of new tokens over the paged 8-bit cache (include/ssba_cache.h).
//
// For one kv head the queries that read it are columns: column j of a sequence
// is (new token j / G, query head j % G).  A wave holds R tiles of 16 columns
// and walks the keys in steps of 32 (two groups of 16 tokens):
//   S^T = K Q^T        v_mfma_f32_16x16x32_bf16, A = 16 keys, B = 16 columns
//   p = exp2(scale_k S - m)
//   O^T += V^T (scale_v p)^T   A = 16 channels, B = 16 columns, 32 keys
// A lane's 4 + 4 scores of a column (keys 4 g + i of both groups, g = lane/16)
// are its B operand of the second product as they are, and the pages keep the
// codes in the A operands' order, so K and V go from memory to registers in
// fully coalesced 16-byte loads and never through the LDS.  A step's codes
// (D 128: 8 KB) are loaded while the step before is computed.  e4m3 codes are
// exact in bf16 (v_cvt_scalef32_pk_bf16_fp8).
// The page numbers and scales of 64 groups are loaded at once, one group per
// lane, and read back with v_readlane: no load waits on another in the loop.
// No maximum is taken in most steps: a column's m stays until a lane's sum of
// probabilities exceeds 2^20 (the scores have outgrown m), a column has none
// yet or keys are masked; then m is raised and the step's probabilities are
// formed again.  What m lags behind is harmless in fp32 and bf16.
// bf16: V's page scale is added in the exponent (log2) instead of multiplying
// every probability; the lane's sum is divided by it again.
// Probabilities: two bf16 terms (16 bits) where few columns leave the matrix
// unit idle.  Elsewhere one fp16 term (11 bits), codes being exact in fp16 too:
// the rounding stays below that of a bf16 output.  fp16 ends at 2^16, so m is
// taken of the weights p * vs there, 2^8 below the largest, and raised when a
// lane's sum of four passes 2^15; weights of less than 2^-22 of the largest are
// held in steps of 2^-32 of it.  Sums of probabilities are relative to the same
// m; where V's scales differ by more than 2^40 they are formed apart, as p * vs
// may be too small for fp32 where p is not.  A chunk of 4096 tokens over 16384
// keys, D 128, takes 478 us and is off by 0.00167 (rms, of which the output's
// own rounding is 0.00166); with one bf16 term 460 us and 0.00236, with two
// 613 us.  The selected chunk: 59.7 us in all, 58.6, 69.
//
// What bounds it, and what it reaches (launch alone):
//   few columns   the pages' bytes: 64 sequences of 8 to 16 thousand tokens, 4 kv
//                 heads, D 128: 122 us, 5.4 TB/s (659 MB, three sets of inputs
//                 in turn; row sums read 6.05 TB/s).  Three waves a SIMD with one
//                 step under way each; four (128 registers) take 148 us, two
//                 steps under way as long as one.
//   many columns  matrix and vector work: 4096 tokens x 16 heads over 16384
//                 keys, D 128: 480 us, 1.15 PFLOP/s.  Two waves a SIMD, 64
//                 columns each: their O takes half of the registers, so the
//                 queries stay in the LDS.
//   lists         few columns of a tile are in use, so vector issue.  Where a
//                 wave has a row alone and G is at most 8, a tile is two times
//                 the same 8 columns with other keys (J): half the exponentials.
//                 1024 tokens x 8 kv heads x 20 pages of 32, D 64, G 3: 44 us, 16
//                 TB/s from the L2 (with bf16 probabilities 43; there J 1 took
//                 48 us, J 4 49: registers).
#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>

#include "ssba_cache_common.h"

namespace ssba {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4a4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kMost = 1048576.f;   // a lane's sum of probabilities of a step: 2^20
// Probabilities in fp16, V's scale included: a lane's sum of four, and how far m is below the largest when it is taken.
constexpr float kMostHalf = 32768.f, kBelow = 8.f;
constexpr float kLow = 0x1p40f;      // a V scale that far below another page's: sums are taken apart
constexpr int kNoKey = 0x40000000;   // first token of a group that is not there: behind every sequence

union Frag {
  bf16x8 v;
  bf16x2 p[4];
  halfx8 h;
  halfx2 hp[4];
  uint32_t u[4];
};

__device__ __forceinline__ bf16x2 codes_lo(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
}
__device__ __forceinline__ bf16x2 codes_hi(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
}

__device__ __forceinline__ halfx2 half_codes_lo(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
}
__device__ __forceinline__ halfx2 half_codes_hi(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum over the wave (of the bits of numbers >= 0: of the numbers).
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));   // row_shr 1
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));   // row_bcast 15
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));   // row_bcast 31
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// x 2^d where 2^d may be less than fp32 holds and the product is not.
__device__ __forceinline__ float shrink(float x, float d) {
  const float h = exp2_(0.5f * d);
  return x * h * h;
}

__device__ __forceinline__ int lane_i(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ float lane_f(float v, int l) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l));
}

// x as NS bf16 terms, each the rounding of what the ones before leave.
template <int NS>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&t)[NS]) {
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    t[s] = (__bf16)x;
    x -= (float)t[s];
  }
}

// What a variant is made of.  A workgroup has CG * KP waves: CG column groups,
// each of whose keys KP waves share.  NQ, NP: bf16 terms of a query value and
// of a probability.  QLDS: the queries stay in the LDS, not in registers.
// J: a tile of 16 columns is J times the same 16 / J columns, each with other
// keys.
template <int D_, int R_, int NQ_, int NP_, bool F32_, bool LISTED_, int CG_, int KP_, bool QLDS_, int J_ = 1>
struct Shape {
  static constexpr int D = D_, R = R_, NQ = NQ_, NP = NP_, CG = CG_, KP = KP_, J = J_;
  static constexpr bool F32 = F32_, LISTED = LISTED_, QLDS = QLDS_;
  static constexpr bool HALF = !F32 && NP == 1;   // the second product in fp16
  static constexpr int THREADS = 64 * CG * KP;
  static constexpr int NH = D / 64;   // 64-channel blocks
  static constexpr int NC = D / 16;   // 16-channel tiles of O
  static constexpr int COLS = 16 * R / J;   // columns of a wave
  static_assert(J == 1 || (LISTED && R == 1 && KP == 1 && !QLDS), "");
};

// Writes E consecutive channels of an output row.
template <bool F32, int E>
__device__ __forceinline__ void store_row(void* o, int64_t at, const float* x) {
  if (F32) {
    typedef float f4a4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<f4a4*>(static_cast<float*>(o) + at + e) = f4a4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(o) + at + e) =
          bf16x4{(__bf16)x[e], (__bf16)x[e + 1], (__bf16)x[e + 2], (__bf16)x[e + 3]};
  }
}

// Which item a workgroup (or a part to be joined) belongs to.
struct Item {
  int seq, h, cbase, ncols, tok0;   // cbase: first column of the workgroup; tok0: token of column 0
  SeqView sv;
};

// unit: sequence, or packed row (LISTED).  False: no such row.
template <bool LISTED>
__device__ __forceinline__ bool item_of(const AttendArgs& a, int unit, int lane, Item* it) {
  if (LISTED) {
    if (unit >= a.b.rows || !seq_of_row(a.b, a.c.page_log2, unit, lane, &it->seq, &it->sv)) return false;
  } else {
    it->seq = unit;
    it->sv = seq_view(a.b, a.c.page_log2, unit);
  }
  it->tok0 = LISTED ? unit - it->sv.begin : 0;
  it->ncols = LISTED ? a.group : min(it->sv.n, a.b.max_new) * a.group;
  return true;
}

// Element offset of channel 0 of a column's row in Q or O.
template <bool LISTED>
__device__ __forceinline__ int64_t row_at(const AttendArgs& a, const Item& it, int col, int64_t st, int64_t sh) {
  const int t = LISTED ? 0 : col / a.group;
  return (int64_t)(it.sv.begin + it.tok0 + t) * st + (int64_t)(it.h * a.group + col - t * a.group) * sh;
}

template <typename P>
__global__ __launch_bounds__(P::THREADS, P::R > 1 || (P::D == 128 && (P::J > 1 || (P::F32 && P::KP == 8))) ? 2 : 3) void k_cache_attend(AttendArgs a) {
  constexpr int D = P::D, R = P::R, NQ = P::NQ, NP = P::NP, NH = P::NH, NC = P::NC, J = P::J;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
  const int mine = J > 1 ? n16 / P::COLS : 0;   // which of the J keys' share this lane's column has
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cg = wave % P::CG, kp = wave / P::CG;
  const int page_log2 = a.c.page_log2;
  const int gpp_log2 = page_log2 - 4;   // groups per page

  // Which keys and columns.  With several column tiles to a head, the items of
  // one XCD (blockIdx mod 8) are consecutive, so that the tiles of a head read
  // its keys from one L2.  Causal tiles differ in length, later tokens see
  // more: long ones start first, within a head, or within all heads of the XCD
  // where these come out even (4 prompts of up to 2048 tokens, 16 heads on 4, D
  // 128: 72.6 us, heads one after another 75.1).
  unsigned id = blockIdx.x;
  int split, ct;
  const unsigned heads = (unsigned)a.b.seqs * a.c.kv_heads;
  if (P::QLDS && a.causal && heads % 8 == 0) {
    const unsigned per = heads / 8 * a.splits, i = id / 8, rest = i % per;
    split = rest % a.splits;
    ct = a.col_tiles - 1 - i / per;
    id = id % 8 * (heads / 8) + rest / a.splits;   // (sequence, head)
  } else {
    if (P::QLDS) {
      const unsigned per = gridDim.x / 8, rest = gridDim.x % 8, x = id % 8;
      id = x * per + min(x, rest) + id / 8;
    }
    split = id % a.splits;
    id /= a.splits;
    ct = id % a.col_tiles;
    if (a.causal) ct = a.col_tiles - 1 - ct;
    id /= a.col_tiles;
  }
  const unsigned item = id * a.col_tiles + ct;
  Item it;
  it.h = id % a.c.kv_heads;
  const int unit = id / a.c.kv_heads;
  // LISTED with several column groups: they are rows.
  const bool there = item_of<P::LISTED>(a, P::LISTED ? unit * P::CG + cg : unit, lane, &it);
  if (!there && (P::KP == 1 || P::CG == 1)) return;
  const int cbase = (P::LISTED ? ct : ct * P::CG + cg) * P::COLS;
  if ((P::CG == 1 || P::KP == 1) && cbase >= it.ncols) return;
  if (P::CG > 1 && P::KP > 1 && ct * P::CG * P::COLS >= it.ncols) return;   // the whole workgroup
  const int cend = min(cbase + P::COLS, it.ncols) - 1;   // < cbase: no columns
  auto limit = [&](int tok) { return a.causal ? min(max(it.sv.start + tok + 1, 0), it.sv.len) : it.sv.len; };
  const int minlim = limit(it.tok0 + (P::LISTED ? 0 : cbase / a.group));
  const int maxlim = cend < cbase ? 0 : limit(it.tok0 + (P::LISTED ? 0 : cend / a.group));

  // This lane's columns.
  int lim[R];
  constexpr int QREGS = P::QLDS ? 1 : R;
  Frag q[QREGS][NQ][NH * 2];
  __shared__ u32x4 s_q[P::QLDS ? P::CG * R * NH * 2 * 64 : 1];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int col = cbase + r * 16 + (J > 1 ? n16 % P::COLS : n16);
    const bool in = col <= cend;
    lim[r] = in ? limit(it.tok0 + (P::LISTED ? 0 : col / a.group)) : 0;
    if (P::QLDS && kp != r % P::KP) continue;   // the waves that share columns share the loading
    const int64_t qo = in ? row_at<P::LISTED>(a, it, col, a.q_st, a.q_sh) : 0;
#pragma unroll
    for (int x = 0; x < NH * 2; ++x) {
      const int ch = (x >> 1) * 64 + g * 16 + (x & 1) * 8;
      if (!P::F32) {
        u32x4 w = {0, 0, 0, 0};
        if (in) w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + qo + ch);
        if (P::QLDS) {
          s_q[((cg * R + r) * NH * 2 + x) * 64 + lane] = w;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) q[r % QREGS][0][x].u[e] = w[e];
        }
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 w = {0, 0, 0, 0};
          if (in) w = *reinterpret_cast<const u32x4a4*>(static_cast<const float*>(a.q) + qo + ch + half * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __bf16 t[NQ];
            split_bf16<NQ>(__uint_as_float(w[e]), t);
#pragma unroll
            for (int s = 0; s < NQ; ++s) q[r % QREGS][s][x].v[half * 4 + e] = t[s];
          }
        }
      }
    }
  }
  if (P::QLDS) __syncthreads();
  // J > 1: share j's product has the queries in share j's columns, 0 in the others, so that one tile collects all J.
  Frag qj[J][NQ][NH * 2];
  if (J > 1)
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int ns = 0; ns < NQ; ++ns)
#pragma unroll
        for (int x = 0; x < NH * 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) qj[j][ns][x].u[e] = mine == j ? q[0][ns][x].u[e] : 0u;

  // Groups of 16 keys, and this wave's steps of J times two groups.
  const int32_t* list = nullptr;
  int groups;
  if (P::LISTED) {
    list = a.lists + ((int64_t)(it.sv.begin + it.tok0) * a.c.kv_heads + it.h) * (1 + a.keep);
    groups = min(max(list[0], 0), a.keep) << gpp_log2;
  } else {
    groups = (maxlim + 15) >> 4;
  }
  const int steps = (groups + 2 * J - 1) / (2 * J);
  // Shares that differ by one step at most.
  int s0 = 0, s1 = steps;
  if (!P::LISTED || P::KP > 1) {
    const unsigned parts = a.splits * P::KP, part = split * P::KP + kp;
    const unsigned each = (unsigned)steps / parts, more = steps - each * parts;
    s0 = each * part + min(part, more);
    s1 = s0 + each + (part < more ? 1 : 0);
  }

  const int32_t* table = a.b.table + (int64_t)it.seq * a.b.max_pages;
  const int64_t head_off = ((int64_t)it.h << page_log2) * D;
  int m_page = 0, m_key = 0;    // of group chunk * 64 + lane: page (-1: none) and first token
  float m_ks = 1.f, m_vs = 1.f, m_lv = 0.f;   // its scales; log2 of V's
  uint32_t vs_top = 0;          // largest of V's scales so far, of all lanes (bits)
  bool m_low = false;           // some are far below it
  auto load_chunk = [&](int chunk) {
    const int gr = chunk * 64 + lane;
    int page = -1, key = kNoKey;
    float ks = 1.f, vs = 1.f;
    if (gr < groups) {
      const int at = gr >> gpp_log2;
      const int lp = P::LISTED ? list[1 + at] : at;
      if (lp >= 0 && lp < a.b.max_pages) {
        const int k0 = (lp << page_log2) + ((gr & ((1 << gpp_log2) - 1)) << 4);
        const int p = k0 < maxlim ? table[lp] : -1;
        if (p >= 0 && p < a.c.pages) {
          page = p;
          key = k0;
          const float* sc = a.c.scale + ((int64_t)p * a.c.kv_heads + it.h) * 2;
          ks = sc[0];
          vs = sc[1];
        }
      }
    }
    m_page = page;
    m_key = key;
    m_ks = ks * a.scale_log2;
    m_vs = P::F32 ? vs : 1.f / vs;
    m_lv = P::F32 ? 0.f : __builtin_amdgcn_logf(vs);
    if (P::HALF) {
      vs_top = max(vs_top, wave_max(page < 0 ? 0u : __float_as_uint(vs)));
      m_low = __builtin_amdgcn_ballot_w64(page >= 0 && vs * kLow < __uint_as_float(vs_top)) != 0;
    }
  };
  int chunk = -1;   // 32 / J steps a chunk

  struct Step {
    u32x4 k[2 * J][NH], v[2 * J][NH];
    int key[2];   // J > 1: these four of the lane's share
    float ks[2], vs[2], lv[2];
    int64_t off[2 * J];
    bool low;     // sums are taken apart
  };
  // The group numbers, scales and K codes of step s, then its V codes.
  auto fetch_k = [&](int s, Step& x) {
    if (s * J >> 5 != chunk) {
      chunk = s * J >> 5;
      load_chunk(chunk);
    }
#pragma unroll
    for (int t = 0; t < 2 * J; ++t) {
      const int gr = 2 * J * s + t;
      const int page = lane_i(m_page, gr & 63);
      const int sub = (gr & ((1 << gpp_log2) - 1)) * 16 * D;
      x.off[t] = (int64_t)max(page, 0) * a.c.page_bytes + head_off + sub;
      const uint8_t* kp_ = a.c.k + x.off[t];
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) x.k[t][hh] = *reinterpret_cast<const u32x4*>(kp_ + lane * 16 + hh * 1024);
    }
    x.low = m_low;
#pragma unroll
    for (int t = 0; t < 2; ++t) {   // behind the loads: the scales may still be on their way
      const int l = (2 * J * s + t) & 63;
      if (J > 1) {
        x.key[t] = __shfl(m_key, l + 2 * mine);
        x.ks[t] = __shfl(m_ks, l + 2 * mine);
        x.vs[t] = __shfl(m_vs, l + 2 * mine);
        if (!P::F32) x.lv[t] = __shfl(m_lv, l + 2 * mine);
      } else {
        // Without lists group g begins at token 16 g: a register less to hold.
        x.key[t] = P::LISTED ? lane_i(m_key, l) : lane_i(m_page, l) < 0 ? kNoKey : (2 * s + t) << 4;
        x.ks[t] = lane_f(m_ks, l);
        x.vs[t] = lane_f(m_vs, l);
        if (!P::F32) x.lv[t] = lane_f(m_lv, l);
      }
    }
  };
  auto fetch_v = [&](Step& x) {
#pragma unroll
    for (int t = 0; t < 2 * J; ++t) {
      const uint8_t* vp = a.c.v + x.off[t];
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) x.v[t][hh] = *reinterpret_cast<const u32x4*>(vp + lane * 16 + hh * 1024);
    }
  };

  floatx4 o[R][NC];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[r][c] = {0.f, 0.f, 0.f, 0.f};
  }

  floatx4 s[2][R];
  auto scores = [&](Step& x) {
    if (J > 1 && __builtin_amdgcn_ballot_w64(max(x.key[0], x.key[1]) + 16 > minlim)) {
      // Keys that are not seen become 0: 0 times a NaN would reach the other shares' columns (their sums run over
      // the same tile).  A NaN that is seen makes all of a row's columns NaN anyway.
#pragma unroll
      for (int t = 0; t < 2 * J; ++t)
        if (lane_i(x.key[t & 1], (t >> 1) * P::COLS) + n16 >= maxlim)
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) x.k[t][hh] = u32x4{0, 0, 0, 0};
    }
    // The queries are read from the LDS again each step: hidden from the
    // compiler, which would otherwise keep them in registers and spill.
    int q_at = cg * R * NH * 2 * 64 + lane;
    if (P::QLDS) asm volatile("" : "+v"(q_at));
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Frag k[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const u32x4 w = x.k[2 * j + t][hh];
            k[t].p[0] = codes_lo(w[2 * u]);
            k[t].p[1] = codes_hi(w[2 * u]);
            k[t].p[2] = codes_lo(w[2 * u + 1]);
            k[t].p[3] = codes_hi(w[2 * u + 1]);
          }
#pragma unroll
          for (int ns = NQ - 1; ns >= 0; --ns)
#pragma unroll
            for (int r = 0; r < R; ++r) {
              Frag b;
              if (P::QLDS) {
                const u32x4 w = s_q[q_at + (r * NH * 2 + hh * 2 + u) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) b.u[e] = w[e];
              } else {
                b = J > 1 ? qj[j][ns][hh * 2 + u] : q[r % QREGS][ns][hh * 2 + u];
              }
#pragma unroll
              for (int t = 0; t < 2; ++t)
                s[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    k[t].v, b.v, j + hh + u == 0 && ns == NQ - 1 ? zero : s[t][r], 0, 0, 0);
            }
        }
  };

  bool settled = false;   // every column has a maximum
  auto finish = [&](Step& x) {
    // Some column does not see some key of this step.
    const bool far = max(x.key[0], x.key[1]) + 16 > minlim;
    const bool edge = J > 1 ? __builtin_amdgcn_ballot_w64(far) != 0 : far;
    if (edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[t][r][i] = x.key[t] + 4 * g + i < lim[r] ? s[t][r][i] * x.ks[t] : -INFINITY;
      x.ks[0] = x.ks[1] = 1.f;
    }
    // Probabilities with the maximum so far, and each lane's sum of them.
    Frag p[R][NP];
    float sum[R];
    bool high = false;
    float top;   // of the lane's sums of four
    auto probabilities = [&]() {
      top = 0.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float mu = m[r] == -INFINITY ? 0.f : m[r];
        float half[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // bf16: V's scale 2^lv goes into the exponent and out of the sum again.
          const float shift = P::F32 ? mu : mu - x.lv[t];
          half[t] = 0.f;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            floatx2 e;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              e[w] = exp2_(__builtin_fmaf(s[t][r][2 * i + w], x.ks[t], -shift));
              half[t] = i + w ? half[t] + e[w] : e[w];
              if (P::F32) e[w] *= x.vs[t];
            }
#pragma unroll
            for (int ns = 0; ns < NP; ++ns) {   // both at once: one conversion
              if (P::HALF) {
                p[r][ns].hp[t * 2 + i] = __builtin_convertvector(e, halfx2);
                continue;
              }
              p[r][ns].p[t * 2 + i] = __builtin_convertvector(e, bf16x2);
              if (ns + 1 < NP) {
                e[0] -= (float)p[r][ns].p[t * 2 + i][0];
                e[1] -= (float)p[r][ns].p[t * 2 + i][1];
              }
            }
          }
        }
        sum[r] = P::F32 ? half[0] + half[1] : __builtin_fmaf(half[0], x.vs[0], half[1] * x.vs[1]);
        if (P::HALF) top = fmaxf(fmaxf(top, half[0]), half[1]);
        else high |= sum[r] > kMost;
      }
      if (P::HALF) high = top > kMostHalf;
    };
    probabilities();
    if (edge || (P::HALF && x.low) || !settled || __builtin_amdgcn_ballot_w64(high)) {
      // Some column has no maximum yet, or has outgrown it.
      bool none = false;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mx = fmaxf(mx, P::HALF ? __builtin_fmaf(s[t][r][i], x.ks[t], x.lv[t]) : s[t][r][i] * x.ks[t]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float to = fmaxf(m[r], P::HALF ? mx - kBelow : mx);
        const float f = to > m[r] ? exp2_(m[r] - to) : 1.f;
        l[r] = !P::HALF ? l[r] * f : to > m[r] ? shrink(l[r], m[r] - to) : l[r];
        m[r] = to;
        none |= to == -INFINITY && lim[r] > 0;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] *= f;
      }
      settled = !__builtin_amdgcn_ballot_w64(none);
      // The sum of a page's probabilities is that of its weights p * vs over vs, unless these may be too small for
      // fp32 beside another page's where the probabilities are not (a page of zeros has a V scale of 2^-64).
      const bool low = P::HALF && x.low;
      if (low) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float mu = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) l[r] += exp2_(__builtin_fmaf(s[t][r][i], x.ks[t], -mu));
        }
        x.vs[0] = x.vs[1] = 0.f;   // those below count for nothing
      }
      probabilities();
    }
#pragma unroll
    for (int r = 0; r < R; ++r) l[r] += sum[r];
    if (edge) {
      // What no column sees may hold anything: its codes become 0, so that a
      // zero probability times them is 0.  A NaN that some columns see and
      // others do not is taken out as well and given to those that see it.
      uint32_t some = 0;
#pragma unroll
      for (int t = 0; t < 2 * J; ++t) {
        const int key = J > 1 ? lane_i(x.key[t & 1], (t >> 1) * P::COLS) : x.key[t & 1];
        const int left = min(max(maxlim - key - 4 * g, 0), 4);
        const uint32_t keep = left == 4 ? ~0u : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x.v[t][hh][e] &= keep;
            some |= ((x.v[t][hh][e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
          }
      }
      if (!P::LISTED && __builtin_amdgcn_ballot_w64(some != 0)) {   // lists: all columns see the same
        // 1 where a column sees a key, times 1 where the key's value is NaN (bit
        // arithmetic: comparisons would take a scalar register pair each).
        constexpr uint32_t kOne = 0x3f80;   // bf16
        Frag sees[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int k = x.key[w >> 1] + 4 * g + (w & 1) * 2 - lim[r];   // negative: seen
            sees[r].u[w] = ((uint32_t)(k >> 31) & kOne) | ((uint32_t)((k + 1) >> 31) & (kOne << 16));
          }
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            Frag bad;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const uint32_t w = x.v[t][hh][e];
              const uint32_t nan = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
              x.v[t][hh][e] = w & ~(nan * 0xffu);
              bad.u[2 * t] = ((nan & 1u) | ((nan & 0x100u) << 8)) * kOne;
              bad.u[2 * t + 1] = ((nan >> 16 & 1u) | (nan >> 8 & 0x10000u)) * kOne;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
              const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad.v, sees[r].v, zero, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i)   // hit is 0 or at least 1
                o[r][hh * 4 + e][i] = __uint_as_float(__float_as_uint(o[r][hh * 4 + e][i]) |
                                                      ((uint32_t)(-__float_as_int(hit[i]) >> 31) & 0x7fc00000u));
            }
          }
      }
    }
    if (P::QLDS) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      Frag pj[NP];   // share j's columns, 0 in the others
      if (J > 1)
#pragma unroll
        for (int ns = 0; ns < NP; ++ns)
#pragma unroll
          for (int e = 0; e < 4; ++e) pj[ns].u[e] = mine == j ? p[0][ns].u[e] : 0u;
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          Frag v;
          if (P::HALF) {
            v.hp[0] = half_codes_lo(x.v[2 * j][hh][e]);
            v.hp[1] = half_codes_hi(x.v[2 * j][hh][e]);
            v.hp[2] = half_codes_lo(x.v[2 * j + 1][hh][e]);
            v.hp[3] = half_codes_hi(x.v[2 * j + 1][hh][e]);
          } else {
            v.p[0] = codes_lo(x.v[2 * j][hh][e]);
            v.p[1] = codes_hi(x.v[2 * j][hh][e]);
            v.p[2] = codes_lo(x.v[2 * j + 1][hh][e]);
            v.p[3] = codes_hi(x.v[2 * j + 1][hh][e]);
          }
#pragma unroll
          for (int ns = NP - 1; ns >= 0; --ns)
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const Frag& w = J > 1 ? pj[ns] : p[r][ns];
              o[r][hh * 4 + e] = P::HALF
                                     ? __builtin_amdgcn_mfma_f32_16x16x32_f16(v.h, w.h, o[r][hh * 4 + e], 0, 0, 0)
                                     : __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, w.v, o[r][hh * 4 + e], 0, 0, 0);
            }
        }
    }
  };

  // One step's codes are under way or in use: V comes during the scores, the
  // next K during the softmax and the second product.
  Step x;
  if (s0 < s1) fetch_k(s0, x);
  for (int st = s0; st < s1; ++st) {
    fetch_v(x);
    // The wave in its products goes first, so that the other of its SIMD has
    // its softmax under them.
    if (P::QLDS) __builtin_amdgcn_s_setprio(1);
    scores(x);
    if (P::QLDS) __builtin_amdgcn_s_setprio(0);
    Step y = x;
    if (st + 1 < s1) fetch_k(st + 1, x);
    finish(y);
  }

#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
  }

  if (J > 1) {
    // The shares of a column, scaled to their common maximum (-inf: nothing seen, O and l are 0).
    float mall = m[0];
#pragma unroll
    for (int x = P::COLS; x < 16; x <<= 1) mall = fmaxf(mall, __shfl_xor(mall, x));
    const float f = m[0] == mall ? 1.f : exp2_(m[0] - mall);
    l[0] = !P::HALF ? l[0] * f : m[0] == mall ? l[0] : shrink(l[0], m[0] - mall);
#pragma unroll
    for (int x = P::COLS; x < 16; x <<= 1) l[0] += __shfl_xor(l[0], x);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      o[0][c] *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int x = P::COLS; x < 16; x <<= 1) o[0][c][i] += __shfl_xor(o[0][c][i], x);
    }
  }

  if (P::KP == 1) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int col = cbase + r * 16 + n16;
      if (col > cend || (J > 1 && mine)) continue;
      const int64_t at = row_at<P::LISTED>(a, it, col, a.o_st, a.o_sh) + g * 4;
      const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float w[4] = {o[r][c][0] * inv, o[r][c][1] * inv, o[r][c][2] * inv, o[r][c][3] * inv};
        store_row<P::F32, 4>(a.o, at + c * 16, w);
      }
    }
    return;
  }

  // The shares of the waves that split the keys, 16 columns at a time: every
  // wave puts its O, scaled to the common maximum, into the LDS and TPC
  // threads a column add them up.
  constexpr int LD = D + 4, TPC = 4 * P::KP < D / 4 ? 4 * P::KP : D / 4, E = D / TPC;
  __shared__ float s_o[P::KP > 1 ? P::CG * P::KP * 16 * LD : 1];
  __shared__ float s_m[P::CG][P::KP][16], s_l[P::CG][P::KP][16];
  const int col = threadIdx.x / TPC, ocg = col >> 4, c16 = col & 15, ch = (threadIdx.x % TPC) * E;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r) __syncthreads();
    if (g == 0) {
      s_m[cg][kp][n16] = m[r];
      s_l[cg][kp][n16] = l[r];
    }
    __syncthreads();
    float mall = s_m[cg][0][n16];
#pragma unroll
    for (int w = 1; w < P::KP; ++w) mall = fmaxf(mall, s_m[cg][w][n16]);
    const float f = m[r] == mall ? 1.f : exp2_(m[r] - mall);   // -inf on both sides: nothing seen, O and l are 0
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const floatx4 w = o[r][c] * f;
      *reinterpret_cast<floatx4*>(&s_o[((cg * P::KP + kp) * 16 + n16) * LD + c * 16 + g * 4]) = w;
    }
    __syncthreads();
    if (ocg >= P::CG) continue;   // more threads than 4 channels each need
    float cm = s_m[ocg][0][c16];
#pragma unroll
    for (int w = 1; w < P::KP; ++w) cm = fmaxf(cm, s_m[ocg][w][c16]);
    float sum = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < P::KP; ++w) {
      const float lw = s_l[ocg][w][c16], d = s_m[ocg][w][c16] - cm;
      if (s_m[ocg][w][c16] == cm) sum += lw;
      else sum += P::HALF ? shrink(lw, d) : lw * exp2_(d);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += s_o[((ocg * P::KP + w) * 16 + c16) * LD + ch + e];
    }
    const int cc = (ct * P::CG + ocg) * P::COLS + r * 16 + c16;
    if (cc >= it.ncols) continue;
    if (a.splits > 1) {
      // [item][split][column][D] and the same with (m, l)
      const int64_t slot = (((int64_t)item * a.splits + split) * (P::CG * R) + ocg * R + r) * 16 + c16;
      float* to = a.part + slot * D;
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<floatx4*>(to + ch + e) = floatx4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
      if (ch == 0) {
        float* ml = a.part_ml + slot * 2;
        ml[0] = cm;
        ml[1] = sum;
      }
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= inv;
      store_row<P::F32, E>(a.o, row_at<P::LISTED>(a, it, cc, a.o_st, a.o_sh) + ch, acc);
    }
  }
}

// Joins the parts of split items.  One workgroup for 16 columns and 32
// channels of an item: 8 threads a column take 4 channels each, two sets of
// them every second part.
constexpr int kMaxSplits = 256;

// RC: tiles of 16 columns of an item.
template <int D, int RC, bool F32, bool LISTED>
__global__ __launch_bounds__(256) void k_cache_join(AttendArgs a) {
  constexpr bool HALF = !F32 && !LISTED && RC > 1;
  __shared__ float s_w[kMaxSplits][16];
  __shared__ float s_sum[16];
  __shared__ floatx4 s_acc[128];
  unsigned id = blockIdx.x;
  const int ch32 = id % (D / 32);
  id /= D / 32;
  const int r = id % RC;
  id /= RC;
  const unsigned item = id;
  const int ct = id % a.col_tiles;
  id /= a.col_tiles;
  Item it;
  it.h = id % a.c.kv_heads;
  if (!item_of<LISTED>(a, id / a.c.kv_heads, threadIdx.x & 63, &it)) return;
  const int c0 = ct * 16 * RC + r * 16;
  if (c0 >= it.ncols) return;
  const int64_t slot0 = ((int64_t)item * a.splits * RC + r) * 16;   // part s: + s * RC * 16
  {
    // 16 threads a column: maximum, weights and sum over the parts.
    const int c = threadIdx.x >> 4, j = threadIdx.x & 15;
    const float* ml = a.part_ml + (slot0 + c) * 2;
    const bool in = c0 + c < it.ncols;
    float m = -INFINITY;
    if (in)
      for (int s = j; s < a.splits; s += 16) m = fmaxf(m, ml[(int64_t)s * RC * 32]);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
    float sum = 0.f;
    if (in)
      for (int s = j; s < a.splits; s += 16) {
        const float ms = ml[(int64_t)s * RC * 32];
        const float w = ms == m ? 1.f : exp2_(ms - m);
        s_w[s][c] = w;
        const float l = ml[(int64_t)s * RC * 32 + 1];
        sum += HALF && ms != m ? shrink(l, ms - m) : w * l;
      }
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) sum += __shfl_xor(sum, x);
    if (j == 0) s_sum[c] = sum;
  }
  __syncthreads();
  const int half = threadIdx.x >> 7, t = threadIdx.x & 127, c = t >> 3, ch = ch32 * 32 + (t & 7) * 4;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  const bool in = c0 + c < it.ncols;
  if (in) {
    const float* part = a.part + (slot0 + c) * D + ch;
#pragma unroll 8
    for (int s = half; s < a.splits; s += 2)
      acc += *reinterpret_cast<const floatx4*>(part + (int64_t)s * RC * 16 * D) * s_w[s][c];
  }
  if (half) s_acc[t] = acc;
  __syncthreads();
  if (half || !in) return;
  acc += s_acc[t];
  const float inv = s_sum[c] == 0.f ? 0.f : 1.f / s_sum[c];
  const float w[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
  store_row<F32, 4>(a.o, row_at<LISTED>(a, it, c0 + c, a.o_st, a.o_sh) + ch, w);
}

template <typename P>
hipError_t launch(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  k_cache_attend<P><<<(unsigned)(p.items * p.splits), P::THREADS, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  constexpr int RC = P::LISTED ? P::R : P::CG * P::R;
  k_cache_join<P::D, RC, P::F32, P::LISTED><<<(unsigned)(p.items * RC * (P::D / 32)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  const bool f32 = dtype == SSBA_DT_F32;
  // D, R, NQ, NP, fp32, lists, column groups, waves that share keys, queries in the LDS, shares of a tile
  switch (p.kind) {
    case kAttendRows:
      if (f32) return launch<Shape<D, 1, 3, 3, true, true, 4, 1, false>>(a, p, s);
      return a.group <= 8 ? launch<Shape<D, 1, 1, 1, false, true, 4, 1, false, 2>>(a, p, s)
                          : launch<Shape<D, 1, 1, 1, false, true, 4, 1, false>>(a, p, s);
    case kAttendRow:
      if (p.threads == 512)
        return f32 ? launch<Shape<D, 1, 3, 3, true, true, 1, 8, false>>(a, p, s)
                   : launch<Shape<D, 1, 1, 2, false, true, 1, 8, false>>(a, p, s);
      return f32 ? launch<Shape<D, 1, 3, 3, true, true, 1, 4, false>>(a, p, s)
                 : launch<Shape<D, 1, 1, 2, false, true, 1, 4, false>>(a, p, s);
    default:
      if (p.threads == 512 && p.tiles == 1)
        return f32 ? launch<Shape<D, 1, 3, 3, true, false, 1, 8, false>>(a, p, s)
                   : launch<Shape<D, 1, 1, 2, false, false, 1, 8, false>>(a, p, s);
      if (f32)
        return p.tiles == 1 ? launch<Shape<D, 1, 3, 3, true, false, 1, 4, false>>(a, p, s)
                            : launch<Shape<D, 1, 3, 3, true, false, 2, 2, false>>(a, p, s);
      switch (p.tiles) {
        case 1: return launch<Shape<D, 1, 1, 2, false, false, 1, 4, false>>(a, p, s);
        case 2:
          return p.threads == 512 ? launch<Shape<D, 2, 1, 1, false, false, 1, 8, false>>(a, p, s)
                                  : launch<Shape<D, 2, 1, 1, false, false, 1, 4, false>>(a, p, s);
        case 4: return launch<Shape<D, 4, 1, 1, false, false, 1, 8, true>>(a, p, s);
        case 8: return launch<Shape<D, 4, 1, 1, false, false, 2, 4, true>>(a, p, s);
        default: return launch<Shape<D, 4, 1, 1, false, false, 4, 2, true>>(a, p, s);
      }
  }
}

}  // namespace

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  return a.c.head_dim == 64 ? launch_d<64>(a, p, dtype, s) : launch_d<128>(a, p, dtype, s);
}

}  // namespace ssba
