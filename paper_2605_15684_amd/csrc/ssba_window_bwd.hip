// Causal attention with a sliding window and sinks, backward
// (include/ssba_window.h).
//
//   k_window_dq     a workgroup has 128 queries, 32 a wave, as the forward: it
//                   forms delta = rowsum(do o) and the log-sum-exp in log2 units
//                   of its rows (kept for the key side), then per key tile
//                   S^T = K Q^T, P = exp2(c S - lse2), dS^T = P (V dO^T - delta),
//                   dQ^T += K^T dS^T
//   k_window_dkdv   a workgroup has 128 keys, 32 a wave, and walks the queries
//                   that see some of them, head after head of the group:
//                   S = Q K^T, dV^T += dO^T P, dS = P (dO V^T - delta),
//                   dK^T += Q^T dS.  Keys that are sinks are seen by every later
//                   query: their queries are cut into chunks.  Where there are
//                   few tiles, several workgroups share the heads of a group
//                   and the queries.
//   k_window_join   adds up the parts of chunks and shares, in their order.
//
// S and dP are formed twice, on either side: one pass that also added dQ would
// need atomics, whose order changes results, or dQ in as many parts as key tiles.
// fp32 as in the forward.  bf16 at D 128 holds dK, dV and V of 32 keys in
// registers and K as operands in the LDS, with tiles of 32 queries: two waves a
// SIMD (K in registers as well leaves one).
//
// Measured, and what bounds it.  bf16, 2 x 8192, 16 heads on 4, D 128, window 2048
// + 16: dq 390 us, dkdv 555, join 6 (with the forward 1120 a call): 930 and 870
// TFLOP/s of what the two compute; matrix units are busy 58 and 55 %, the rest are
// exponentials, masks and conversions that overlap only in part, and waits for the
// LDS.  2 x 200 rows, 4 heads, D 64: 11.4 and 11.4 us, chains of a few tiles.
// fp32, packed 6269 rows, 6 heads on 2, D 128, window 512: 180, 200 and 12 us; one
// wave a SIMD, and a second turn of few workgroups (the chip is busy 49 and 59 %
// of the time, the matrix units 40 % of that).
//
// What a query does not see must not reach it, nor it what it does not see, and
// 0 times a NaN would: where a result is not finite, the workgroup computes once
// more with the tiles that are seen in part taken row by row.  So it does where a
// row's log-sum-exp is very large (kFar).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ssba_common.h"
#include "ssba_window_tiles.h"

namespace ssba {
namespace {

// Reads of the LDS run AHEAD ahead of the products that use them, READS for every
// two: with two waves a SIMD a product that waits for its own read leaves the
// matrix cores idle.
template <class T, int AHEAD, int READS>
__device__ __forceinline__ void order_rows() {
  if constexpr (T::ORDERED) {
    __builtin_amdgcn_sched_group_barrier(kDsRead, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, READS / 2, 0);
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, READS - READS / 2, 0);
    }
  }
}

// exp2(scale s - lse2).  The scores are the forward's, to the bit, so lse2's own
// rounding is all that takes a probability past 1: by a third at most at 2^20, by
// more than exp2 holds from about 2^28 on, which made infinities of finite inputs.
// Where rows are past kFar the careful passes compute, which bound it by 1.  In us,
// dq and dkdv of 2 x 8192 rows, 16 heads on 4, window 2048, bf16, without a bound,
// as it is, and bounded everywhere: D 128 857, 862, 869; D 64 485, 487, 502.  NaN
// stays NaN (IEEE minimum).
constexpr float kFar = 1048576.f;
template <bool CAREFUL>
__device__ __forceinline__ float probability(float s, float scale, float lse2) {
  const float x = __builtin_fmaf(s, scale, -lse2);
  return __builtin_amdgcn_exp2f(CAREFUL ? __builtin_elementwise_minimum(x, 0.f) : x);
}

// --------------------------------------------------------------------------
// dQ.  delta of the rounded o is off by that rounding, most where a row sees few
// keys.  The sums of ds over a row, which would be 0 with the exact one, say by
// how much: the key side gets it corrected.  Here ds itself is formed with the
// one from o; TERMS 2 (up to 1024 keys a row) makes up for it by not rounding ds
// to 8 bits.  Errors of dq and dk against 64 bits, over that of a result's own
// rounding (window 64, D 64, 200 rows): 1.58 and 1.53 without either, 1.20 and
// 1.42 with both.
// --------------------------------------------------------------------------
template <class T, bool CAREFUL, int TERMS, int G>
__device__ __forceinline__ void dq_pass(const WindowArgs& a, const WPlace& p, int group, int wave, int lane, char* kA,
                                        char* kB, char* vA, char* vB, floatx16 (&acc)[T::NDB], float& delta, float& off,
                                        float& lse2) {
  constexpr int NB = T::NB, NDB = T::NDB;
  const int l32 = lane & 31, hw = lane >> 5;
  const int w0 = p.r0 + 32 * wave, w1 = min(w0 + 31, p.len - 1);
  const int i = w0 + l32;
  const int64_t row = p.begin + min(i, p.len - 1);
  WCopy<T> ck, cv;
  ck.init(a.k, (int64_t)p.b * a.sk.b + (int64_t)p.kvh * a.sk.h + (int64_t)p.begin * a.sk.t, a.sk.t, wave, lane);
  cv.init(a.v, (int64_t)p.b * a.sv.b + (int64_t)p.kvh * a.sv.h + (int64_t)p.begin * a.sv.t, a.sv.t, wave, lane);

  const int last = min(p.r0 + kWindowRows, p.len) - 1;
  const int low = max(p.r0 - a.window + 1, 0) / T::ROWS;
  const int n_sink = min((int)(((unsigned)min(a.sinks, last + 1) + T::ROWS - 1) / T::ROWS), low);
  const int n = (n_sink + last / T::ROWS - low + 1 + G - 1) / G;   // turns: those behind the last tile see nothing
  auto first_of = [&](int turn) {
    const int c = G * turn + group;
    return (c < n_sink ? c : low + c - n_sink) * T::ROWS;
  };
  auto issue = [&](int c, char* kn, char* vn) {
    ck.issue(first_of(c), p.len, kn, wave);
    cv.issue(first_of(c), p.len, vn, wave);
  };
  // The end of a tile's copy.
  auto arrive = [&](char* kn, char* vn) {
    ck.land(kn, wave, lane);
    cv.land(vn, wave, lane);
  };
  auto all_there = [&]() {
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
  };
  issue(0, kA, vA);   // before the rows: all are on their way at once

  const char* gp = static_cast<const char*>(a.dout) + ((int64_t)p.b * a.sdo.b + (int64_t)p.h * a.sdo.h + row * a.sdo.t) * T::SIZE;
  WRow<T> q, g;
  q.load(static_cast<const char*>(a.q) + ((int64_t)p.b * a.sq.b + (int64_t)p.h * a.sq.h + row * a.sq.t) * T::SIZE, hw);
  g.load(gp, hw);
  lse2 = a.lse[((int64_t)p.b * a.heads + p.h) * a.seq + row] * kLog2e;
  delta = 0.f;
  {
    using R = WTile<T::D, T::F32 ? kF32 : kBf16>;   // values as they are
    WRow<R> o, y;
    o.load(static_cast<const char*>(a.o) + ((int64_t)p.b * a.so.b + (int64_t)p.h * a.so.h + row * a.so.t) * T::SIZE, hw);
    y.load(gp, hw);
#pragma unroll
    for (int ks = 0; ks < R::NKS; ++ks)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (T::F32) {
          delta = __builtin_fmaf(o.f[0][ks][e], y.f[0][ks][e], delta);
        } else {
          const uint32_t u = __float_as_uint(o.f[0][ks][e]), v = __float_as_uint(y.f[0][ks][e]);
          delta = __builtin_fmaf(__uint_as_float(u << 16), __uint_as_float(v << 16), delta);
          delta = __builtin_fmaf(__uint_as_float(u & 0xFFFF0000u), __uint_as_float(v & 0xFFFF0000u), delta);
        }
      }
    delta += __shfl_xor(delta, 32);
  }

  WLane<T> at(lane);
  off = 0.f;   // sum of the lane's ds
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = floatx16{};

  auto body = [&](int c, const char* kc, const char* vc, char* kn, char* vn) {
    if (!CAREFUL && c + 1 < n) issue(c + 1, kn, vn);
    const int j0 = first_of(c);
    const bool none = j0 > w1 || (j0 + T::ROWS - 1 <= w0 - a.window && j0 >= a.sinks);
    if (!none) {
      const bool whole = j0 + T::ROWS - 1 <= w0 && (j0 + T::ROWS <= a.sinks || j0 > w0 + 31 - a.window);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
        at.forget();
        floatx16 s = {}, ds;
#pragma unroll
        for (int e = 0; e < 16; ++e) ds[e] = -delta;
        rows_products<T, false>(s, kc + nb * T::HALF, q, ds, vc + nb * T::HALF, g, at);
        order_rows<T, 6, 2>();
#pragma unroll
        for (int e = 0; e < 16; ++e) ds[e] *= probability<CAREFUL>(s[e], a.scale_log2, lse2);
        if (!whole) {
          const uint32_t bits = keys_seen(i, j0 + 32 * nb, a.window, a.sinks) >> (4 * hw);
#pragma unroll
          for (int e = 0; e < 16; ++e) ds[e] = keep_if(bit_of(bits, e), ds[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) off += ds[e];
        if constexpr (CAREFUL) {
          if (!whole) {
            cols_product_seen<T>(
                acc, kc + nb * T::HALF, ds,
                reinterpret_cast<float*>((wave < T::TILE / 4096 ? kn : vn) + 4096 * (wave % (T::TILE / 4096))), lane,
                keys_seen(i, j0 + 32 * nb, a.window, a.sinks));
            continue;
          }
        }
        cols_product<T, TERMS>(acc, kc + nb * T::HALF, ds, at);
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (!CAREFUL && c + 1 < n) arrive(kn, vn);
    all_there();
  };

  arrive(kA, vA);
  all_there();
  if constexpr (CAREFUL) {   // one tile at a time: the other buffers are room for the rows' weights
    for (int c = 0; c < n; ++c) {
      body(c, kA, vA, kB, vB);
      if (c + 1 == n) break;
      issue(c + 1, kA, vA);
      arrive(kA, vA);
      all_there();
    }
  } else {
    for (int c = 0; c < n; c += 2) {
      body(c, kA, vA, kB, vB);
      if (c + 1 < n) body(c + 1, kB, vB, kA, vA);
    }
  }
  off += __shfl_xor(off, 32);
}

// T: tiles of the first pass; TC: of the careful one.  G: groups of four waves
// that share the key tiles.
template <class T, class TC, int TERMS, int G>
__global__ __launch_bounds__(256 * G, T::SPLIT && T::D == 128 ? 1 : 2) void k_window_dq(WindowArgs a) {
  constexpr int NDB = T::NDB, BYTES = T::TILE > TC::TILE ? T::TILE : TC::TILE;
  __shared__ __attribute__((aligned(16))) char kA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char kB[G][BYTES];
  __shared__ __attribute__((aligned(16))) char vA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char vB[G][BYTES];
  __shared__ float s_off[G == 1 ? 1 : 256];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, hw = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4;
  const int group = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  WPlace p;
  if (!place_query(a, lane, &p)) return;
  const int i = p.r0 + 32 * wave + (lane & 31);
  const bool in = i < p.len;
  const int64_t row = p.begin + min(i, p.len - 1);
  const int64_t to = ((int64_t)p.b * a.heads + p.h) * a.seq + row;

  floatx16 acc[NDB];
  float delta, off, lse2;
  if (threadIdx.x == 0) s_bad = 0;
  dq_pass<T, false, TERMS, G>(a, p, group, wave, lane, kA[group], kB[group], vA[group], vB[group], acc, delta, off, lse2);
  const bool far = fabsf(lse2) > kFar;
  if (__builtin_amdgcn_ballot_w64(in && (far || not_finite<NDB>(acc))) && lane == 0) s_bad = 1;
  __syncthreads();
  if (s_bad)
    dq_pass<TC, true, TERMS, G>(a, p, group, wave, lane, kA[group], kB[group], vA[group], vB[group], acc, delta, off, lse2);
  if constexpr (G == 2) {
    const int thread = threadIdx.x & 255;
    if (group) s_off[thread] = off;
    join_groups<NDB>(acc, group, thread, kA[0], kB[0], vA[0], vB[0]);
    if (!group) off += s_off[thread];
  }
  if (!in) return;
  if (hw == 0 && group == 0) {
    a.ndelta[to] = -(delta + off);
    a.lse2[to] = lse2;
  }
  char* dq = static_cast<char*>(a.dq) + ((int64_t)p.b * a.sdq.b + (int64_t)p.h * a.sdq.h + row * a.sdq.t) * T::SIZE;
  store_cols<T, NDB / G>(dq + group * (NDB / G) * 32 * T::SIZE, acc, a.scale, hw);
}

// --------------------------------------------------------------------------
// dK, dV
// --------------------------------------------------------------------------

// What a workgroup of the key side does: 128 keys of a kv head, and the queries
// q0 .. q1 - 1 of its sequence of the group's heads g0 .. g1 - 1.
struct KeyPlace {
  int b, kvh, begin, len, k0, q0, q1, g0, g1;
  int64_t part;   // where its parts go, -1: it has all queries of all heads
};

// Slot of a sequence's chunk 0, as place_slot counts tiles.
__device__ __forceinline__ int chunk_slot(const WindowArgs& a, int begin, int s) { return begin / a.chunk + s; }

// The part-th of `parts` of the queries, in multiples of 32; none: q0 = q1.
__device__ __forceinline__ void share_queries(int parts, int part, KeyPlace* p) {
  if (parts == 1) return;
  const int all = p->q1 - p->q0, each = ((all + parts - 1) / parts + 31) / 32 * 32;
  const int from = min((int64_t)part * each, (int64_t)all), to = min((int64_t)from + each, (int64_t)all);
  p->q1 = p->q0 + to;
  p->q0 += from;
}

__device__ __forceinline__ bool place_keys(const WindowArgs& a, int lane, KeyPlace* p) {
  const unsigned units = (unsigned)a.batch * a.kv_heads, cut = (unsigned)a.sink_tiles * a.chunk_slots;
  const unsigned shares = a.head_parts * a.query_parts, per = (a.slots + cut) * shares;
  unsigned id = blockIdx.x, unit, at;
  if (a.spread) {
    unit = id % units;
    at = id / units;
  } else {
    id = xcd_order(id, units * per);
    unit = id / per;
    at = id % per;
  }
  const int share = at % shares, heads = share % a.head_parts, part = share / a.head_parts;
  at /= shares;
  p->g0 = heads * a.group / a.head_parts;
  p->g1 = (heads + 1) * a.group / a.head_parts;
  p->b = unit / a.kv_heads;
  p->kvh = unit % a.kv_heads;
  const unsigned kept = cut + (shares > 1 ? a.slots : 0);   // tiles and chunks that leave parts
  p->part = at < kept ? (((int64_t)unit * kept + at) * shares + share) * 2 * kWindowRows : -1;
  if (at >= cut) {   // a tile of keys; its queries, or the first chunk of them, end with the window
    WPlace w;
    if (!place_slot(a, at - cut, lane, &w)) return false;
    p->begin = w.begin;
    p->len = w.len;
    p->k0 = w.r0;
    p->q0 = w.r0;
    if (w.r0 < a.sinks) {
      if (a.chunk_slots) return false;   // its chunks have workgroups of their own
      p->q1 = w.len;
    } else {
      p->q1 = a.window < w.len - w.r0 - kWindowRows ? w.r0 + kWindowRows - 1 + a.window : w.len;
    }
    share_queries(a.query_parts, part, p);
    return true;
  }
  const int tile = at / a.chunk_slots, slot = at % a.chunk_slots;
  int s = 0, c = slot;
  if (a.cu) {
    s = seq_of_slot(a.cu, a.seqs, a.seq, a.chunk, slot, lane);
    seq_rows(a, s, &p->begin, &p->len);
    c = slot - chunk_slot(a, p->begin, s);
  } else {
    p->begin = 0;
    p->len = a.seq;
  }
  p->k0 = tile * kWindowRows;
  if (c < 0 || p->k0 >= p->len) return false;
  const int64_t q0 = p->k0 + (int64_t)c * a.chunk;
  if (q0 >= p->len) return false;
  p->q0 = (int)q0;
  p->q1 = p->len - p->q0 < a.chunk ? p->len : p->q0 + a.chunk;
  share_queries(a.query_parts, part, p);
  return true;
}

// 64 floats into the LDS, those from n on as 0.
__device__ __forceinline__ void copy_values(const float* from, int n, float* dst, int lane) {
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), (short)0, 4 * n, kRawBufferFlags);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)dst, 4, 4 * lane, 0, 0, 0);
}

template <class T, bool CAREFUL, int G>
__device__ __forceinline__ void dkdv_pass(const WindowArgs& a, const KeyPlace& p, int group, int wave, int lane, char* s_k,
                                          char* qA, char* qB, char* gA, char* gB, float (*rA)[64], float (*rB)[64],
                                          int* s_bad, floatx16 (&dk)[T::NDB], floatx16 (&dv)[T::NDB]) {
  constexpr int NB = T::NB, NDB = T::NDB;
  // The wave's keys as operands in the LDS where registers are short.
  constexpr bool KLDS = T::ORDERED;
  const int l32 = lane & 31, hw = lane >> 5;
  const int w0 = p.k0 + 32 * wave, w1 = min(w0 + 31, p.len - 1);   // the wave's keys
  const int j = w0 + l32;

  WCopy<T> cq, cg;
  cq.init(a.q, (int64_t)p.b * a.sq.b + ((int64_t)p.kvh * a.group + p.g0) * a.sq.h + (int64_t)p.begin * a.sq.t, a.sq.t, wave,
          lane);
  cg.init(a.dout, (int64_t)p.b * a.sdo.b + ((int64_t)p.kvh * a.group + p.g0) * a.sdo.h + (int64_t)p.begin * a.sdo.t,
          a.sdo.t, wave, lane);
  const int64_t head = (int64_t)p.b * a.heads + p.kvh * a.group + p.g0;
  const char* q_base = cq.base;
  const char* g_base = cg.base;
  const float* l_base = a.lse2 + head * a.seq + p.begin;
  const float* d_base = a.ndelta + head * a.seq + p.begin;

  // Every G-th tile of queries, head after head: as many for each group (one behind the last tile of a head sees
  // nothing).
  const int t0 = p.q0 / T::ROWS, tiles = (p.q1 - 1) / T::ROWS - t0 + 1;
  const int per_head = (tiles + G - 1) / G * G, n = per_head / G * (p.g1 - p.g0);
  int next_g = 0, next_t = group;   // of the tile that is copied next
  auto issue = [&](char* qd, char* gd, float (*rd)[64]) {
    cq.base = q_base + (int64_t)next_g * a.sq.h * T::SIZE;
    cg.base = g_base + (int64_t)next_g * a.sdo.h * T::SIZE;
    const int i0 = (t0 + next_t) * T::ROWS;
    cq.issue(i0, p.len, qd, wave);
    cg.issue(i0, p.len, gd, wave);
    if (wave < 2) copy_values((wave ? d_base : l_base) + (int64_t)next_g * a.seq + i0, max(min(p.len - i0, T::ROWS), 0), rd[wave], lane);
    if ((next_t += G) >= per_head) {
      next_t = group;
      ++next_g;
    }
  };

  // The end of a tile's copy.
  auto arrive = [&](char* qn, char* gn) {
    cq.land(qn, wave, lane);
    cg.land(gn, wave, lane);
  };
  auto all_there = [&]() {
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
  };
  issue(qA, gA, rA);   // before the keys: all are on their way at once

  using KRow = typename std::conditional<KLDS, WRowLds<T>, WRow<T>>::type;
  KRow k;
  WRow<T> v;
  {
    const int64_t row = p.begin + min(j, p.len - 1);
    WRow<T> kr;
    kr.load(static_cast<const char*>(a.k) + ((int64_t)p.b * a.sk.b + (int64_t)p.kvh * a.sk.h + row * a.sk.t) * T::SIZE, hw);
    if constexpr (KLDS) {   // read by this wave alone
      k.at = s_k + 1024 * T::NKS * wave + 16 * lane;
#pragma unroll
      for (int ks = 0; ks < T::NKS; ++ks)
        *reinterpret_cast<floatx4*>(s_k + 1024 * (T::NKS * wave + ks) + 16 * lane) = kr.f[0][ks];
    } else {
      k = kr;
    }
    v.load(static_cast<const char*>(a.v) + ((int64_t)p.b * a.sv.b + (int64_t)p.kvh * a.sv.h + row * a.sv.t) * T::SIZE, hw);
  }
  WLane<T> place(lane);
  int at = group;   // tile of the head
#pragma unroll
  for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = floatx16{};

  auto body = [&](int c, const char* qc, const char* gc, float (*rc)[64], char* qn, char* gn, float (*rn)[64]) {
    if (!CAREFUL && c + 1 < n) issue(qn, gn, rn);
    const int i0 = (t0 + at) * T::ROWS;
    if ((at += G) >= per_head) at = group;
    const bool none = i0 + T::ROWS - 1 < w0 || (G > 1 && i0 >= p.q1) || (w1 <= i0 - a.window && w0 >= a.sinks) || w0 >= p.len;
    if (!none) {
      if (!CAREFUL && __builtin_amdgcn_ballot_w64(fabsf(rc[0][lane]) > kFar)) *s_bad = 1;   // some row of the tile
      const bool whole = i0 >= max(w0 + 31, p.q0) && i0 + T::ROWS <= p.q1 &&
                         (w0 + 32 <= a.sinks || w0 > i0 + T::ROWS - 1 - a.window);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
        place.forget();
        floatx16 pr = {}, ds;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const floatx4 d = *reinterpret_cast<const floatx4*>(&rc[1][32 * nb + 2 * e + 4 * hw]);
#pragma unroll
          for (int x = 0; x < 4; ++x) ds[e + x] = d[x];
        }
        rows_products<T, true>(pr, qc + nb * T::HALF, k, ds, gc + nb * T::HALF, v, place);
        order_rows<T, 8, 3>();
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const floatx4 l = *reinterpret_cast<const floatx4*>(&rc[0][32 * nb + 2 * e + 4 * hw]);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            pr[e + x] = probability<CAREFUL>(pr[e + x], a.scale_log2, l[x]);
            ds[e + x] *= pr[e + x];
          }
        }
        if (!whole) {
          const uint32_t bits = queries_seeing(j, i0 + 32 * nb, p.q0, p.q1, a.window, a.sinks) >> (4 * hw);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t seen = bit_of(bits, e);
            pr[e] = keep_if(seen, pr[e]);
            ds[e] = keep_if(seen, ds[e]);
          }
        }
        if constexpr (CAREFUL) {
          if (!whole) {
            float* room = reinterpret_cast<float*>((wave < T::TILE / 4096 ? qn : gn) + 4096 * (wave % (T::TILE / 4096)));
            const uint32_t bits = queries_seeing(j, i0 + 32 * nb, p.q0, p.q1, a.window, a.sinks);
            cols_product_seen<T>(dv, gc + nb * T::HALF, pr, room, lane, bits);
            cols_product_seen<T>(dk, qc + nb * T::HALF, ds, room, lane, bits);
            continue;
          }
        }
        cols_product<T>(dv, gc + nb * T::HALF, pr, place);
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
        cols_product<T>(dk, qc + nb * T::HALF, ds, place);
        if constexpr (T::ORDERED) __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (!CAREFUL && c + 1 < n) arrive(qn, gn);
    all_there();
  };

  arrive(qA, gA);
  all_there();
  if constexpr (CAREFUL) {   // one tile at a time: the other buffers are room for the rows' weights
    for (int c = 0; c < n; ++c) {
      body(c, qA, gA, rA, qB, gB, rB);
      if (c + 1 == n) break;
      issue(qA, gA, rA);
      arrive(qA, gA);
      all_there();
    }
  } else {
    for (int c = 0; c < n; c += 2) {
      body(c, qA, gA, rA, qB, gB, rB);
      if (c + 1 < n) body(c + 1, qB, gB, rB, qA, gA, rA);
    }
  }
}

// T: tiles of the first pass; TC: of the careful one.  G: groups of four waves
// that share the tiles of queries.
template <class T, class TC, int G>
__global__ __launch_bounds__(256 * G, T::SPLIT && T::D == 128 ? 1 : 2) void k_window_dkdv(WindowArgs a) {
  constexpr int NDB = T::NDB, BYTES = T::TILE > TC::TILE ? T::TILE : TC::TILE;
  __shared__ __attribute__((aligned(16))) char s_k[T::ORDERED ? G * 4 * T::NKS * 1024 : 16];
  __shared__ __attribute__((aligned(16))) char qA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char qB[G][BYTES];
  __shared__ __attribute__((aligned(16))) char gA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char gB[G][BYTES];
  __shared__ __attribute__((aligned(16))) float rA[G][2][64];   // lse2, -delta of the tile's rows
  __shared__ __attribute__((aligned(16))) float rB[G][2][64];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, l32 = lane & 31, hw = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4;
  const int group = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  KeyPlace p;
  if (!place_keys(a, lane, &p)) return;
  const int j = p.k0 + 32 * wave + l32;
  const bool in = j < p.len;
  floatx16 dk[NDB], dv[NDB];
  if (threadIdx.x == 0) s_bad = 0;
  char* keys = s_k + (T::ORDERED ? group * 4 * T::NKS * 1024 : 0);
  if (p.q0 < p.q1) {
    dkdv_pass<T, false, G>(a, p, group, wave, lane, keys, qA[group], qB[group], gA[group], gB[group], rA[group], rB[group],
                           &s_bad, dk, dv);
    if (__builtin_amdgcn_ballot_w64(in && (not_finite<NDB>(dk) || not_finite<NDB>(dv))) && lane == 0) s_bad = 1;
    __syncthreads();
    if (s_bad)
      dkdv_pass<TC, true, G>(a, p, group, wave, lane, keys, qA[group], qB[group], gA[group], gB[group], rA[group], rB[group],
                             &s_bad, dk, dv);
  } else {
#pragma unroll
    for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = floatx16{};
  }
  if constexpr (G == 2) {
    join_groups<NDB>(dk, group, threadIdx.x & 255, qA[0], qB[0], gA[0], gB[0]);
    join_groups<NDB>(dv, group, threadIdx.x & 255, qA[0], qB[0], gA[0], gB[0]);
  }
  if (!in) return;
  const int ch = group * (NDB / G) * 32;   // first channel
  if (p.part >= 0) {
    using P = WTile<T::D, kF32>;
    char* to = reinterpret_cast<char*>(a.part + (p.part + 32 * wave + l32) * T::D + ch);
    store_cols<P, NDB / G>(to, dk, 1.f, hw);
    store_cols<P, NDB / G>(to + (int64_t)kWindowRows * T::D * 4, dv, 1.f, hw);
    return;
  }
  const int64_t row = p.begin + j;
  store_cols<T, NDB / G>(
      static_cast<char*>(a.dk) + ((int64_t)p.b * a.sdk.b + (int64_t)p.kvh * a.sdk.h + row * a.sdk.t + ch) * T::SIZE, dk,
      a.scale, hw);
  store_cols<T, NDB / G>(
      static_cast<char*>(a.dv) + ((int64_t)p.b * a.sdv.b + (int64_t)p.kvh * a.sdv.h + row * a.sdv.t + ch) * T::SIZE, dv,
      1.f, hw);
}

// Adds up the parts of a tile's chunks and shares, in their order: a workgroup
// has a tile's 2048 / D rows, 8 channels a thread.  Of a tile that is cut into
// chunks the first chunk's does all.
template <class T>
__global__ __launch_bounds__(256) void k_window_join(WindowArgs a) {
  constexpr int D = T::D, ROWS = 2048 / D, PARTS = kWindowRows / ROWS;
  const int lane = threadIdx.x & 63;
  unsigned id = blockIdx.x;
  const int sub = id % PARTS;
  id /= PARTS;
  const int shares = a.head_parts * a.query_parts;
  const unsigned cut = (unsigned)a.sink_tiles * a.chunk_slots, kept = cut + (shares > 1 ? a.slots : 0);
  const unsigned unit = id / kept, at = id % kept;
  int begin = 0, len = a.seq, k0, parts = shares;
  if (at >= cut) {
    WPlace w;
    if (!place_slot(a, at - cut, lane, &w)) return;
    if (a.chunk_slots && w.r0 < a.sinks) return;
    begin = w.begin;
    len = w.len;
    k0 = w.r0;
  } else {
    const int tile = at / a.chunk_slots, slot = at % a.chunk_slots;
    if (a.cu) {
      const int s = seq_of_slot(a.cu, a.seqs, a.seq, a.chunk, slot, lane);
      seq_rows(a, s, &begin, &len);
      if (slot != chunk_slot(a, begin, s)) return;
    } else if (slot) {
      return;
    }
    k0 = tile * kWindowRows;
    if (k0 >= len) return;
    parts *= (len - k0 + a.chunk - 1) / a.chunk;
  }
  const int r = sub * ROWS + (int)threadIdx.x / (D / 8), ch = (int)threadIdx.x % (D / 8) * 8;
  if (k0 + r >= len) return;
  const float* from = a.part + (((int64_t)unit * kept + at) * shares * 2 * kWindowRows + r) * D + ch;
  const int b = unit / a.kv_heads, kvh = unit % a.kv_heads;
  const int64_t row = begin + k0 + r;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < parts; ++c) {
      const float* x = from + ((int64_t)c * 2 + which) * kWindowRows * D;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const floatx4 y = *reinterpret_cast<const floatx4*>(x + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[4 * h + e] += y[e];
      }
    }
    const Strides& st = which ? a.sdv : a.sdk;
    char* to = static_cast<char*>(which ? a.dv : a.dk) + ((int64_t)b * st.b + (int64_t)kvh * st.h + row * st.t + ch) * T::SIZE;
    const float f = which ? 1.f : a.scale;
    if constexpr (T::F32) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<floatx4*>(to + 16 * h) =
            floatx4{sum[4 * h] * f, sum[4 * h + 1] * f, sum[4 * h + 2] * f, sum[4 * h + 3] * f};
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(pack2(sum[0] * f, sum[1] * f), pack2(sum[2] * f, sum[3] * f),
                                                 pack2(sum[4] * f, sum[5] * f), pack2(sum[6] * f, sum[7] * f));
    }
  }
}

// T: tiles of the query side, TK: of the key side; TC: of the careful passes
// (the key side's in those of TK where it is bf16).
template <class T, class TC, int TERMS>
void launch_dq(const WindowArgs& a, hipStream_t s) {
  const unsigned groups = (unsigned)((int64_t)a.batch * a.heads * a.slots);
  if constexpr (!(T::SPLIT && T::D == 128))
    if (share_tiles(a, groups)) return k_window_dq<T, TC, TERMS, 2><<<groups, 512, 0, s>>>(a);
  k_window_dq<T, TC, TERMS, 1><<<groups, 256, 0, s>>>(a);
}

template <class T, class TK, class TC>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  using TKC = typename std::conditional<T::F32, TC, TK>::type;
  const int64_t units = (int64_t)a.batch * a.kv_heads, cut = (int64_t)a.sink_tiles * a.chunk_slots;
  const int64_t shares = (int64_t)a.head_parts * a.query_parts, kept = cut + (shares > 1 ? a.slots : 0);
  if (!T::F32 && (int64_t)a.window + a.sinks <= 1024)
    launch_dq<T, TC, T::F32 ? 1 : 2>(a, s);
  else
    launch_dq<T, TC, 1>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned groups = (unsigned)(units * (a.slots + cut) * shares);
  bool few = false;
  if constexpr (!(T::SPLIT && T::D == 128)) {
    few = share_tiles(a, groups, T::SPLIT ? 1024 : 256);
    if (few) k_window_dkdv<TK, TKC, 2><<<groups, 512, 0, s>>>(a);
  }
  if (!few) k_window_dkdv<TK, TKC, 1><<<groups, 256, 0, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess || !kept) return e;
  k_window_join<T><<<(unsigned)(units * kept * (kWindowRows * T::D / 2048)), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const WindowArgs& a, int dtype, hipStream_t s) {
  using Split = WTile<D, kF32Split>;
  using Half = WTile<D, kBf16>;
  if (dtype == SSBA_DT_F32) return launch<Split, Split, WTile<D, kF32>>(a, s);
  return launch<Half, WTile<D, kBf16, D == 128 ? 1 : 2>, Half>(a, s);
}

}  // namespace

hipError_t launch_window_backward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s) {
  return head_dim == 64 ? launch_d<64>(a, dtype, s) : launch_d<128>(a, dtype, s);
}

}  // namespace ssba
