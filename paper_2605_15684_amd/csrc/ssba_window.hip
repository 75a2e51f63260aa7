// Causal attention with a sliding window and sinks, forward
// (include/ssba_window.h).
//
// A workgroup has 128 consecutive queries of one head, 32 a wave, and walks the
// key tiles that some of them see: those with sinks, then those of the window.
// K and V tiles are copied to the LDS while the tile before is computed.
//   S^T = K Q^T, p = exp2(scale log2(e) S - m), O^T += V^T p^T
// so that a lane has 16 keys of one query and the probabilities are the second
// product's operand as they are.  m is raised only where a lane's sum of
// probabilities passes 2^20, or a query has none yet; it may lag behind
// otherwise, which is harmless in fp32 and bf16.
//
// 32 queries a wave is what a 32 x 32 product takes, so that K and V are read
// from the LDS once for 32; tiles of 64 keys (bf16) leave two workgroups a CU.
// Partly seen tiles take their mask from a word of bits a lane, made once a tile.
// The wave in its second products goes first (s_setprio): the other one of its
// SIMD has exponentials to do then (16384 tokens below: 185 to 177 us).
//
// fp32: values are split into three bf16 terms on their way to the LDS, and six
// of the nine pairs of terms multiplied: 192 cycles where v_mfma_f32_32x32x2_f32
// takes 512 (packed, 5 sequences, 6 heads on 2, D 64: 43.6 to 32.8 us).
//
// Measured, and what bounds it.  bf16, 16384 tokens, 16 heads on 4, D 128, window
// 1024 + 4: 167 us a call, 800 TFLOP/s of what the rows see; the matrix units are
// busy 46 % of the time and vector instructions issue in 41 %, which overlap only
// in part at two waves a SIMD (the registers allow no more).  2 x 8192, window
// 2048: 290 us, matrix units 52 %.  fp32, D 64, 5 sequences of up to 1101, window
// 333: 25 us, one workgroup a CU that waits for its own tiles.  fp32, D 128: one
// wave a SIMD; 318 workgroups leave the chip half empty in their second turn (130
// us, matrix units 37 % where they run).
//
// A value that a query does not see must not reach it, and 0 times a NaN would:
// where a result is not finite, the workgroup computes once more with the tiles
// that some query sees in part taken row by row.  So it does where the sum of a
// query's probabilities is far off: the rounding of scores past 2^29 can do it.
#include <hip/hip_runtime.h>

#include "ssba_common.h"
#include "ssba_window_tiles.h"

namespace ssba {
namespace {

constexpr float kMost = 1048576.f;   // a lane's sum of probabilities of a half tile: 2^20
constexpr float kLeast = 0x1p-60f;   // see k_window_forward
constexpr float kLn2 = 0.69314718055994530942f;

// x y - z, not fused.
__device__ __forceinline__ float two_roundings(float x, float y, float z) {
#pragma clang fp contract(off)
  const float xy = x * y;
  return xy - z;
}

// The wave's queries over every G-th key tile from the `group`-th on.  CAREFUL:
// one tile at a time, the other buffers are room for the rows' weights.
template <class T, bool CAREFUL, int G>
__device__ __forceinline__ void forward_pass(const WindowArgs& a, const WPlace& p, int group, int wave, int lane, char* kA,
                                             char* kB, char* vA, char* vB, floatx16 (&o)[T::NDB], float& m, float& l) {
  constexpr int NB = T::NB, NDB = T::NDB;
  const int l32 = lane & 31, hw = lane >> 5;
  const int w0 = p.r0 + 32 * wave, w1 = min(w0 + 31, p.len - 1);   // the wave's queries; w1 < w0: none
  const int i = w0 + l32;
  const bool in = i < p.len;

  WCopy<T> ck, cv;
  ck.init(a.k, (int64_t)p.b * a.sk.b + (int64_t)p.kvh * a.sk.h + (int64_t)p.begin * a.sk.t, a.sk.t, wave, lane);
  cv.init(a.v, (int64_t)p.b * a.sv.b + (int64_t)p.kvh * a.sv.h + (int64_t)p.begin * a.sv.t, a.sv.t, wave, lane);

  // Tiles 0 .. n_sink - 1, then those of the window.
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
  issue(0, kA, vA);   // before the queries: both are on their way at once

  WRow<T> q;
  q.load(static_cast<const char*>(a.q) +
             ((int64_t)p.b * a.sq.b + (int64_t)p.h * a.sq.h + (int64_t)(p.begin + min(i, p.len - 1)) * a.sq.t) * T::SIZE,
         hw);
  WLane<T> at(lane);
  bool settled = false;
  const float scale = a.scale_log2;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int db = 0; db < NDB; ++db) o[db] = floatx16{};

  auto body = [&](int c, const char* kc, const char* vc, char* kn, char* vn) {
    if (!CAREFUL && c + 1 < n) issue(c + 1, kn, vn);
    const int j0 = first_of(c);
    const bool none = j0 > w1 || (j0 + T::ROWS - 1 <= w0 - a.window && j0 >= a.sinks);
    if (!none) {
      const bool whole = j0 + T::ROWS - 1 <= w0 && (j0 + T::ROWS <= a.sinks || j0 > w0 + 31 - a.window);
      floatx16 s[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        s[nb] = floatx16{};
        rows_product<T>(s[nb], kc + nb * T::HALF, q, at);
      }
      if (!whole) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint32_t bits = keys_seen(i, j0 + 32 * nb, a.window, a.sinks) >> (4 * hw);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint32_t seen = bit_of(bits, e);
            s[nb][e] = __uint_as_float((__float_as_uint(s[nb][e]) & seen) | (0xFF800000u & ~seen));   // -infinity
          }
        }
      }
      floatx16 pr[NB];
      float sum[NB];
      auto probabilities = [&]() {
        const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          sum[nb] = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            // With the product rounded as m's is, the largest of all gives 1 at any size of the scores (past 2^31 their
            // rounding alone is beyond what exp2 takes).
            const float x = CAREFUL ? two_roundings(s[nb][e], scale, mu) : __builtin_fmaf(s[nb][e], scale, -mu);
            pr[nb][e] = __builtin_amdgcn_exp2f(x);
            sum[nb] += pr[nb][e];
          }
        }
      };
      bool high = !settled;
      if (settled) {
        probabilities();
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) high |= sum[nb] > kMost;
      }
      if (__builtin_amdgcn_ballot_w64(high)) {
        float mx = -INFINITY;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[nb][e]);
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale;
        const float to = fmaxf(m, mx);
        const float f = to > m ? __builtin_amdgcn_exp2f(m - to) : 1.f;
        m = to;
        l *= f;
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[db] *= f;
        settled = !__builtin_amdgcn_ballot_w64(m == -INFINITY && in);
        probabilities();
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) l += sum[nb];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (CAREFUL) {
          if (!whole) {
            cols_product_seen<T>(
                o, vc + nb * T::HALF, pr[nb],
                reinterpret_cast<float*>((wave < T::TILE / 4096 ? kn : vn) + 4096 * (wave % (T::TILE / 4096))), lane,
                keys_seen(i, j0 + 32 * nb, a.window, a.sinks));
            continue;
          }
        }
        cols_product<T>(o, vc + nb * T::HALF, pr[nb], at);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    if (!CAREFUL && c + 1 < n) arrive(kn, vn);
    all_there();
  };

  arrive(kA, vA);
  all_there();
  if constexpr (CAREFUL) {
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
}

// T: tiles of the first pass; TC: of the careful one.  G: groups of four waves
// that share the key tiles.
template <class T, class TC, int G>
__global__ __launch_bounds__(256 * G, T::SPLIT && T::D == 128 ? 1 : 2) void k_window_forward(WindowArgs a) {
  constexpr int NDB = T::NDB, BYTES = T::TILE > TC::TILE ? T::TILE : TC::TILE;
  __shared__ __attribute__((aligned(16))) char kA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char kB[G][BYTES];
  __shared__ __attribute__((aligned(16))) char vA[G][BYTES];
  __shared__ __attribute__((aligned(16))) char vB[G][BYTES];
  __shared__ float s_ml[G == 1 ? 1 : 2 * G][256];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, hw = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % 4;
  const int group = G == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  WPlace p;
  if (!place_query(a, lane, &p)) return;
  const int i = p.r0 + 32 * wave + (lane & 31);
  const bool in = i < p.len;
  floatx16 o[NDB];
  float m, l;
  if (threadIdx.x == 0) s_bad = 0;
  forward_pass<T, false, G>(a, p, group, wave, lane, kA[group], kB[group], vA[group], vB[group], o, m, l);
  // At least about 1, and 2^20 of each lane and half tile at most, but for what m's own rounding does.
  const float all = l + __shfl_xor(l, 32);
  const bool off = (G == 1 || m != -INFINITY) && !(all > kLeast && all < 1.f / kLeast);
  if (__builtin_amdgcn_ballot_w64(in && (off || not_finite<NDB>(o))) && lane == 0) s_bad = 1;
  __syncthreads();
  if (s_bad) forward_pass<TC, true, G>(a, p, group, wave, lane, kA[group], kB[group], vA[group], vB[group], o, m, l);

  l += __shfl_xor(l, 32);
  if constexpr (G == 2) {
    const int thread = threadIdx.x & 255;
    s_ml[2 * group][thread] = m;
    s_ml[2 * group + 1][thread] = l;
    __syncthreads();
    const float m2 = s_ml[2 - 2 * group][thread], l2 = s_ml[3 - 2 * group][thread], top = fmaxf(m, m2);
    const float f = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), f2 = m2 == top ? 1.f : __builtin_amdgcn_exp2f(m2 - top);
    m = top;
    l = l * f + l2 * f2;
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] *= f;
    join_groups<NDB>(o, group, thread, kA[0], kB[0], vA[0], vB[0]);
  }
  if (!in) return;
  const int64_t row = p.begin + i;
  char* to = static_cast<char*>(a.o) + ((int64_t)p.b * a.so.b + (int64_t)p.h * a.so.h + row * a.so.t) * T::SIZE;
  store_cols<T, NDB / G>(to + group * (NDB / G) * 32 * T::SIZE, o, 1.f / l, hw);
  if (a.lse && hw == 0 && group == 0)
    a.lse[((int64_t)p.b * a.heads + p.h) * a.seq + row] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <class T, class TC>
hipError_t launch(const WindowArgs& a, hipStream_t s) {
  const unsigned groups = (unsigned)((int64_t)a.batch * a.heads * a.slots);
  if constexpr (!(T::SPLIT && T::D == 128)) {
    if (share_tiles(a, groups)) {
      k_window_forward<T, TC, 2><<<groups, 512, 0, s>>>(a);
      return hipGetLastError();
    }
  }
  k_window_forward<T, TC, 1><<<groups, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const WindowArgs& a, int dtype, hipStream_t s) {
  if (dtype == SSBA_DT_F32) return launch<WTile<D, kF32Split>, WTile<D, kF32>>(a, s);
  return launch<WTile<D, kBf16>, WTile<D, kBf16>>(a, s);
}

}  // namespace

hipError_t launch_window_forward(const WindowArgs& a, int head_dim, int dtype, hipStream_t s) {
  return head_dim == 64 ? launch_d<64>(a, dtype, s) : launch_d<128>(a, dtype, s);
}

}  // namespace ssba
