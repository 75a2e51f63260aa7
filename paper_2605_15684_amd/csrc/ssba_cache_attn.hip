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
// The maximum m is raised only when a score exceeds it by 2^kSlack: p stays
// below 2^kSlack, whose products and sums fp32 holds, and most steps need no
// reduction across lanes.
#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>

#include "ssba_cache.h"

namespace ssba {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4a4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kSlack = 16.0f;
constexpr int kNoKey = 0x40000000;   // first token of a group that is not there: behind every sequence

union Frag {
  bf16x8 v;
  bf16x2 p[4];
  uint32_t u[4];
};

__device__ __forceinline__ bf16x2 codes_lo(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
}
__device__ __forceinline__ bf16x2 codes_hi(uint32_t w) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

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

// NS: bf16 terms of a query value and of a probability (1: bf16 tensors, 3: fp32).
template <int D, int R, int NS, bool LISTED, bool BY_COLUMNS>
__global__ __launch_bounds__(256, R == 1 ? 3 : 2) void k_cache_attend(AttendArgs a) {
  constexpr int NH = D / 64;   // 64-channel blocks
  constexpr int NC = D / 16;   // 16-channel tiles of O
  constexpr int COLS = 16 * R;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int page_log2 = a.c.page_log2;
  const int gpp_log2 = page_log2 - 4;   // groups per page

  // Which keys and columns.
  unsigned id = blockIdx.x;
  int split = 0;
  if (!BY_COLUMNS) {
    split = id % a.splits;
    id /= a.splits;
  }
  const int ct = id % a.col_tiles;
  id /= a.col_tiles;
  const int h = id % a.c.kv_heads;
  const int unit = id / a.c.kv_heads;
  int seq, row0 = 0;
  if (LISTED) {
    row0 = BY_COLUMNS ? unit * 4 + wave : unit;
    seq = row0 < a.b.rows ? seq_of_row(a.b, row0, lane) : a.b.seqs;
    if (seq >= a.b.seqs) return;
  } else {
    seq = unit;
  }
  const SeqView sv = seq_view(a.b, page_log2, seq);
  int cbase, ncols, tok0;   // first column, columns, first token
  if (LISTED) {
    tok0 = row0 - sv.begin;
    if (tok0 < 0 || tok0 >= sv.n) return;
    cbase = ct * COLS;
    ncols = a.group;
  } else {
    tok0 = 0;
    cbase = (BY_COLUMNS ? ct * 4 + wave : ct) * COLS;
    ncols = min(sv.n, a.b.max_new) * a.group;
  }
  // Waves that share keys stay together for the merge; cbase is the workgroup's then.
  if (cbase >= ncols) return;
  const int cend = min(cbase + COLS, ncols) - 1;
  const int before = sv.len - sv.n;   // tokens in front of the new ones
  auto limit = [&](int tok) { return a.causal ? min(max(before + tok + 1, 0), sv.len) : sv.len; };
  const int minlim = limit(tok0 + (LISTED ? 0 : cbase / a.group));
  const int maxlim = limit(tok0 + (LISTED ? 0 : cend / a.group));

  // This lane's columns.
  int lim[R];
  int64_t orow[R];
  Frag q[R][NS][NH * 2];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int col = cbase + r * 16 + n16;
    const bool there = col <= cend;
    const int tok = tok0 + (LISTED ? 0 : col / a.group);
    const int head = h * a.group + (LISTED ? col : col % a.group);
    lim[r] = there ? limit(tok) : 0;
    orow[r] = there ? (int64_t)(sv.begin + tok) * a.o_st + (int64_t)head * a.o_sh : -1;
    const int64_t qo = (int64_t)(sv.begin + tok) * a.q_st + (int64_t)head * a.q_sh;
#pragma unroll
    for (int x = 0; x < NH * 2; ++x) {
      const int ch = (x >> 1) * 64 + g * 16 + (x & 1) * 8;
      if (NS == 1) {
        u32x4 w = {0, 0, 0, 0};
        if (there) w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + qo + ch);
#pragma unroll
        for (int e = 0; e < 4; ++e) q[r][0][x].u[e] = w[e];
      } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          u32x4 w = {0, 0, 0, 0};
          if (there) w = *reinterpret_cast<const u32x4a4*>(static_cast<const float*>(a.q) + qo + ch + half * 4);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __bf16 t[NS];
            split_bf16<NS>(__uint_as_float(w[e]), t);
#pragma unroll
            for (int s = 0; s < NS; ++s) q[r][s][x].v[half * 4 + e] = t[s];
          }
        }
      }
    }
  }

  // Groups of 16 keys, and this wave's steps of two groups.
  const int32_t* list = nullptr;
  int groups;
  if (LISTED) {
    list = a.lists + ((int64_t)row0 * a.c.kv_heads + h) * (1 + a.keep);
    groups = min(max(list[0], 0), a.keep) << gpp_log2;
  } else {
    groups = (maxlim + 15) >> 4;
  }
  const int steps = (groups + 1) >> 1;
  int s0 = 0, s1 = steps;
  if (!BY_COLUMNS) {
    const int parts = a.splits * 4, part = split * 4 + wave;
    s0 = (int)((int64_t)steps * part / parts);
    s1 = (int)((int64_t)steps * (part + 1) / parts);
  }

  const int32_t* table = a.b.table + (int64_t)seq * a.b.max_pages;
  const int64_t head_off = ((int64_t)h << page_log2) * D;
  int m_page = 0, m_key = 0;    // of group chunk * 64 + lane: page (-1: none) and first token
  float m_ks = 1.f, m_vs = 1.f;
  auto load_chunk = [&](int chunk) {
    const int gr = chunk * 64 + lane;
    int page = -1, key = kNoKey;
    float ks = 1.f, vs = 1.f;
    if (gr < groups) {
      const int at = gr >> gpp_log2;
      const int lp = LISTED ? list[1 + at] : at;
      if (lp >= 0 && lp < a.b.max_pages) {
        const int k0 = (lp << page_log2) + ((gr & ((1 << gpp_log2) - 1)) << 4);
        const int p = k0 < maxlim ? table[lp] : -1;
        if (p >= 0 && p < a.c.pages) {
          page = p;
          key = k0;
          const float* sc = a.c.scale + ((int64_t)p * a.c.kv_heads + h) * 2;
          ks = sc[0];
          vs = sc[1];
        }
      }
    }
    m_page = page;
    m_key = key;
    m_ks = ks;
    m_vs = vs;
  };

  struct Step {
    u32x4 k[2][NH], v[2][NH];
    int key[2];
    float ks[2], vs[2];
  };
  auto fetch = [&](int s, Step& x) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int l = (2 * s + t) & 63;
      const int page = lane_i(m_page, l);
      x.key[t] = lane_i(m_key, l);
      x.ks[t] = lane_f(m_ks, l);
      x.vs[t] = lane_f(m_vs, l);
      const int sub = ((2 * s + t) & ((1 << gpp_log2) - 1)) * 16 * D;
      const int64_t off = (int64_t)max(page, 0) * a.c.page_bytes + head_off + sub;
      const uint8_t* kp = a.c.k + off + lane * 16;
      const uint8_t* vp = a.c.v + off + lane * 16;
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) {
        x.k[t][hh] = *reinterpret_cast<const u32x4*>(kp + hh * 1024);
        x.v[t][hh] = *reinterpret_cast<const u32x4*>(vp + hh * 1024);
      }
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

  auto compute = [&](Step& x) {
    floatx4 s[2][R];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[t][r] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Frag k;
          k.p[0] = codes_lo(x.k[t][hh][2 * u]);
          k.p[1] = codes_hi(x.k[t][hh][2 * u]);
          k.p[2] = codes_lo(x.k[t][hh][2 * u + 1]);
          k.p[3] = codes_hi(x.k[t][hh][2 * u + 1]);
#pragma unroll
          for (int ns = NS - 1; ns >= 0; --ns)
#pragma unroll
            for (int r = 0; r < R; ++r)
              s[t][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k.v, q[r][ns][hh * 2 + u].v, s[t][r], 0, 0, 0);
        }
    }
    // Some column does not see some key of this step.
    const bool edge = max(x.key[0], x.key[1]) + 16 > minlim;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float c = x.ks[t] * a.scale_log2;
#pragma unroll
      for (int r = 0; r < R; ++r) s[t][r] *= c;
    }
    if (edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (x.key[t] + 4 * g + i >= lim[r]) s[t][r][i] = -INFINITY;
    }
    bool raise = false;
    float top[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = s[0][r][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[r] = fmaxf(top[r], s[t][r][i]);
      raise |= top[r] > m[r] + kSlack;
    }
    if (__builtin_amdgcn_ballot_w64(raise)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float mx = fmaxf(top[r], __shfl_xor(top[r], 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float to = fmaxf(m[r], mx);
        const float f = to > m[r] ? exp2_(m[r] - to) : 1.f;
        m[r] = to;
        l[r] *= f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] *= f;
      }
    }
    Frag p[R][NS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mu = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = exp2_(s[t][r][i] - mu);
          l[r] += e;
          __bf16 terms[NS];
          split_bf16<NS>(e * x.vs[t], terms);
#pragma unroll
          for (int ns = 0; ns < NS; ++ns) p[r][ns].v[t * 4 + i] = terms[ns];
        }
    }
    if (edge) {
      // What no column sees may hold anything: its codes become 0, so that a
      // zero probability times them is 0.  A NaN that some columns see and
      // others do not is taken out as well and given to those that see it.
      uint32_t some = 0;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int left = min(max(maxlim - x.key[t] - 4 * g, 0), 4);
        const uint32_t keep = left == 4 ? ~0u : (1u << (8 * left)) - 1u;
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x.v[t][hh][e] &= keep;
            some |= ((x.v[t][hh][e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
          }
      }
      if (__builtin_amdgcn_ballot_w64(some != 0)) {
        Frag sees[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sees[r].v[t * 4 + i] = (__bf16)(x.key[t] + 4 * g + i < lim[r] ? 1.f : 0.f);
#pragma unroll
        for (int hh = 0; hh < NH; ++hh)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            Frag bad;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              uint32_t w = x.v[t][hh][e];
              const uint32_t nan = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
              w &= ~(nan * 0xffu);
              x.v[t][hh][e] = w;
#pragma unroll
              for (int i = 0; i < 4; ++i) bad.v[t * 4 + i] = (__bf16)((nan >> (8 * i)) & 1u ? 1.f : 0.f);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
              const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad.v, sees[r].v, zero, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (hit[i] > 0.f) o[r][hh * 4 + e][i] = NAN;
            }
          }
      }
    }
#pragma unroll
    for (int hh = 0; hh < NH; ++hh)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        Frag v;
        v.p[0] = codes_lo(x.v[0][hh][e]);
        v.p[1] = codes_hi(x.v[0][hh][e]);
        v.p[2] = codes_lo(x.v[1][hh][e]);
        v.p[3] = codes_hi(x.v[1][hh][e]);
#pragma unroll
        for (int ns = NS - 1; ns >= 0; --ns)
#pragma unroll
          for (int r = 0; r < R; ++r)
            o[r][hh * 4 + e] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.v, p[r][ns].v, o[r][hh * 4 + e], 0, 0, 0);
      }
  };

  Step x, y;
  int chunk = s0 >> 5;   // 32 steps a chunk
  if (s0 < s1) {
    load_chunk(chunk);
    fetch(s0, x);
  }
  auto next = [&](int s, Step& to) {
    if (s >= s1) return;
    if ((s >> 5) != chunk) {
      chunk = s >> 5;
      load_chunk(chunk);
    }
    fetch(s, to);
  };
  for (int s = s0; s < s1; s += 2) {
    next(s + 1, y);
    compute(x);
    if (s + 1 >= s1) break;
    next(s + 2, x);
    compute(y);
  }

#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
  }

  if (BY_COLUMNS) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (orow[r] < 0) continue;
      const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const floatx4 w = o[r][c] * inv;
        if (NS == 1) {
          __bf16* to = static_cast<__bf16*>(a.o) + orow[r] + c * 16 + g * 4;
          typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
          *reinterpret_cast<bf16x4*>(to) = bf16x4{(__bf16)w[0], (__bf16)w[1], (__bf16)w[2], (__bf16)w[3]};
        } else {
          typedef float f4a4 __attribute__((ext_vector_type(4), aligned(4)));
          *reinterpret_cast<f4a4*>(static_cast<float*>(a.o) + orow[r] + c * 16 + g * 4) = w;
        }
      }
    }
    return;
  }

  // The four waves' shares of the keys, 16 columns at a time: every wave puts
  // its O, scaled to the common maximum, into the LDS and 16 threads a column
  // add them up.
  constexpr int LD = D + 4;
  __shared__ float s_o[4][16][LD];
  __shared__ float s_m[4][16], s_l[4][16];
  const int col = threadIdx.x >> 4, ch = (threadIdx.x & 15) * (D / 16);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r) __syncthreads();
    if (g == 0) {
      s_m[wave][n16] = m[r];
      s_l[wave][n16] = l[r];
    }
    __syncthreads();
    const float mall = fmaxf(fmaxf(s_m[0][n16], s_m[1][n16]), fmaxf(s_m[2][n16], s_m[3][n16]));
    const float f = m[r] == mall ? 1.f : exp2_(m[r] - mall);   // -inf on both sides: nothing seen, O and l are 0
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const floatx4 w = o[r][c] * f;
      *reinterpret_cast<floatx4*>(&s_o[wave][n16][c * 16 + g * 4]) = w;
    }
    __syncthreads();
    const float cm = fmaxf(fmaxf(s_m[0][col], s_m[1][col]), fmaxf(s_m[2][col], s_m[3][col]));
    float sum = 0.f, acc[D / 16];
#pragma unroll
    for (int e = 0; e < D / 16; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      sum += s_l[w][col] * (s_m[w][col] == cm ? 1.f : exp2_(s_m[w][col] - cm));
#pragma unroll
      for (int e = 0; e < D / 16; ++e) acc[e] += s_o[w][col][ch + e];
    }
    const int cc = cbase + r * 16 + col;
    if (cc > cend) continue;
    if (a.splits > 1) {
      float* to = a.part + (((int64_t)blockIdx.x * R + r) * 16 + col) * (D + 2);
#pragma unroll
      for (int e = 0; e < D / 16; ++e) to[ch + e] = acc[e];
      if (ch == 0) {
        to[D] = cm;
        to[D + 1] = sum;
      }
    } else {
      const int tok = tok0 + (LISTED ? 0 : cc / a.group);
      const int head = h * a.group + (LISTED ? cc : cc % a.group);
      const int64_t oo = (int64_t)(sv.begin + tok) * a.o_st + (int64_t)head * a.o_sh + ch;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) {
        if (NS == 1) static_cast<__bf16*>(a.o)[oo + e] = (__bf16)(acc[e] * inv);
        else static_cast<float*>(a.o)[oo + e] = acc[e] * inv;
      }
    }
  }
}

// Joins the parts of split items: 16 threads a column, one workgroup per item
// and 16 columns.
template <int D, int R, bool F32, bool LISTED>
__global__ __launch_bounds__(256) void k_cache_join(AttendArgs a) {
  unsigned id = blockIdx.x;
  const int r = id % R;
  id /= R;
  const unsigned item = id;
  const int ct = id % a.col_tiles;
  id /= a.col_tiles;
  const int h = id % a.c.kv_heads;
  const int unit = id / a.c.kv_heads;
  const int seq = LISTED ? seq_of_row(a.b, unit, threadIdx.x & 63) : unit;
  if (seq >= a.b.seqs) return;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int tok0 = LISTED ? unit - sv.begin : 0;
  if (LISTED && (tok0 < 0 || tok0 >= sv.n)) return;
  const int ncols = LISTED ? a.group : min(sv.n, a.b.max_new) * a.group;
  const int col = threadIdx.x >> 4, ch = (threadIdx.x & 15) * (D / 16);
  const int cc = ct * 16 * R + r * 16 + col;
  if (cc >= ncols) return;
  const float* part = a.part + (((int64_t)item * a.splits * R + r) * 16 + col) * (D + 2);
  const int64_t stride = (int64_t)R * 16 * (D + 2);
  float m = -INFINITY;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, part[s * stride + D]);
  float sum = 0.f, acc[D / 16];
#pragma unroll
  for (int e = 0; e < D / 16; ++e) acc[e] = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float* p = part + s * stride;
    const float f = p[D] == m ? 1.f : exp2_(p[D] - m);
    sum += p[D + 1] * f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) acc[e] += p[ch + e] * f;
  }
  const int tok = tok0 + (LISTED ? 0 : cc / a.group);
  const int head = h * a.group + (LISTED ? cc : cc % a.group);
  const int64_t oo = (int64_t)(sv.begin + tok) * a.o_st + (int64_t)head * a.o_sh + ch;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < D / 16; ++e) {
    if (F32) static_cast<float*>(a.o)[oo + e] = acc[e] * inv;
    else static_cast<__bf16*>(a.o)[oo + e] = (__bf16)(acc[e] * inv);
  }
}

template <int D, int R, int NS, bool LISTED>
hipError_t launch(const AttendArgs& a, const AttendPlan& p, hipStream_t s) {
  if (p.by_columns) {
    k_cache_attend<D, R, NS, LISTED, true><<<(unsigned)p.items, 256, 0, s>>>(a);
  } else {
    k_cache_attend<D, R, NS, LISTED, false><<<(unsigned)(p.items * p.splits), 256, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.splits > 1) k_cache_join<D, R, NS == 3, LISTED><<<(unsigned)(p.items * R), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  if (dtype == SSBA_DT_F32)
    return p.listed ? launch<D, 1, 3, true>(a, p, s) : launch<D, 1, 3, false>(a, p, s);
  if (p.listed) return launch<D, 1, 1, true>(a, p, s);
  switch (p.tiles16) {
    case 1: return launch<D, 1, 1, false>(a, p, s);
    case 2: return launch<D, 2, 1, false>(a, p, s);
    default: return launch<D, 4, 1, false>(a, p, s);
  }
}

}  // namespace

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int dtype, hipStream_t s) {
  return a.c.head_dim == 64 ? launch_d<64>(a, p, dtype, s) : launch_d<128>(a, p, dtype, s);
}

}  // namespace ssba
