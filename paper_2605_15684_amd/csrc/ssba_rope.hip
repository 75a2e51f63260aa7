// Rotary positions with several axes (include/ssba_rope.h).
//
// A workgroup takes 4 tokens: its threads form the cosines and sines of their
// pairs (one per thread at D 128), leave them in the LDS and then turn the
// heads, each thread the same pairs of one token in every few heads, with those
// pairs' cosines and sines in registers.  So an angle costs one sine in 64 bits
// for all heads; the rest is one pass over the data, 16 bytes a lane and
// neighbouring lanes on neighbouring bytes (two rows of fp32 chunks instead of 32
// bytes a lane: 48.8 to 43.2 us below).  The first heads' values are loaded before
// the angles are formed, four heads are under way at once.
//
// Bound by HBM: 16384 tokens of 24 + 8 heads, bf16, D 128, 45 us in a trace (6.0
// TB/s); of 16 + 16 heads, fp32, D 64, 43 (6.2).  Few tokens: a chain of loads, angle,
// barrier and store, 4.4 us of 8 tokens (their heads shared by several
// workgroups), less than the 10 us that the call costs the host.
//
// Angles: x = pos * freq in quarter turns, reduced to |r| <= 1/2 by x - rint(x)
// in 64 bits (one rounding, of the fused multiply-add), then the Taylor series
// of the sine and cosine of r pi/2, whose first terms left out are below 2e-11
// and 2e-10 of 1.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "ssba_rope_common.h"

namespace ssba {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr float kStays = 2.f;   // in a cosine's place: the pair stays as it is

// cos and sin of pos * f quarter turns.
__device__ __forceinline__ float2 turn(int pos, double f, bool inverse) {
  const double p = (double)pos;
  const double n = __builtin_rint(p * f);
  const double r = __builtin_fma(p, f, -n) * 1.57079632679489661923;
  const double z = r * r;
  double s = -1.0 / 39916800, c = -1.0 / 3628800;   // -1/11!, -1/10!
  s = __builtin_fma(s, z, 1.0 / 362880);
  c = __builtin_fma(c, z, 1.0 / 40320);
  s = __builtin_fma(s, z, -1.0 / 5040);
  c = __builtin_fma(c, z, -1.0 / 720);
  s = __builtin_fma(s, z, 1.0 / 120);
  c = __builtin_fma(c, z, 1.0 / 24);
  s = __builtin_fma(s, z, -1.0 / 6);
  c = __builtin_fma(c, z, -0.5);
  s = __builtin_fma(s * z, r, r);
  c = __builtin_fma(c, z, 1.0);
  // n mod 4, of an n that may be far outside int.
  const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const double sn = q & 1 ? c : s, cs = q & 1 ? s : c;
  const float sine = (float)(q & 2 ? -sn : sn), cosine = (float)((q + 1) & 2 ? -cs : cs);
  return make_float2(cosine, inverse ? -sine : sine);
}

__device__ __forceinline__ void turn_pair(float& a, float& b, float2 w) {
  const float x = __builtin_fmaf(a, w.x, -(b * w.y)), y = __builtin_fmaf(b, w.x, a * w.y);
  a = w.x == kStays ? a : x;
  b = w.x == kStays ? b : y;
}

// Sixteen bytes of a row (fp32 rows may begin at any multiple of 4 bytes).
template <bool F32>
struct Chunk {
  static constexpr int N = F32 ? 4 : 8;   // channels
  typedef float vec4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef typename std::conditional<F32, vec4, floatx4>::type vec;
  floatx4 v;
  __device__ __forceinline__ void load(const char* p) { v = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void store(char* p) const { *reinterpret_cast<vec*>(p) = v; }
  __device__ __forceinline__ void get(float (&x)[N]) const {
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = v[j];
    } else {
      const floatx8 y = __builtin_convertvector(__builtin_bit_cast(bf16x8, v), floatx8);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = y[j];
    }
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    if constexpr (F32) {
      v = floatx4{x[0], x[1], x[2], x[3]};
    } else {
      v = __builtin_bit_cast(floatx4, __builtin_convertvector(floatx8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}, bf16x8));
    }
  }
};

// One workgroup: kRopeRows tokens, a part of the heads.  A thread holds a chunk
// of a row, or two, D/2 channels apart (HALVES: each other's partners; fp32).
template <int D, bool F32, bool HALVES>
__global__ __launch_bounds__(256) void k_rope(TurnArgs a) {
  constexpr int R = kRopeRows, H2 = D / 2, N = Chunk<F32>::N, E = HALVES || F32 ? 2 : 1;
  constexpr int PER = N * E / 2;   // pairs of a thread
  constexpr int TPR = H2 / PER, SLOTS = 256 / (TPR * R), SIZE = F32 ? 4 : 2;
  constexpr int U = 4;   // heads of a thread under way at once
  __shared__ float2 s_turn[R][H2];
  const int64_t tok0 = (int64_t)(blockIdx.x / a.head_parts) * R;
  const int part = blockIdx.x % a.head_parts;
  const int at = threadIdx.x % TPR, row = threadIdx.x / TPR % R, slot = threadIdx.x / (TPR * R);
  const int64_t tok = tok0 + row;
  const bool in = tok < a.tokens;
  const int64_t b = in ? tok / a.rows : 0, t = in ? tok - b * a.rows : 0;
  const int all = a.heads[0] + a.heads[1];
  const int each = (all + a.head_parts - 1) / a.head_parts;
  const int h_end = in ? min(all, (part + 1) * each) : 0;
  const int ch = at * N;
  const int64_t x0 = b * a.x_sb[0] + t * a.x_st[0] + ch, x1 = b * a.x_sb[1] + t * a.x_st[1] + ch;
  const int64_t y0 = b * a.y_sb[0] + t * a.y_st[0] + ch, y1 = b * a.y_sb[1] + t * a.y_st[1] + ch;

  Chunk<F32> v[U][E];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * SLOTS;
      if (h >= h_end) continue;
      const bool second = h >= a.heads[0];
      const char* p = a.x[second] + (second ? x1 + (h - a.heads[0]) * a.x_sh[1] : x0 + h * a.x_sh[0]) * SIZE;
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e].load(p + e * H2 * SIZE);
    }
  };
  int h = part * each + slot;
  load(h);

  for (int i = threadIdx.x; i < R * H2; i += 256) {
    const int r = i / H2, j = i % H2;
    const int64_t tk = tok0 + r;
    float2 w = make_float2(kStays, 0.f);
    const int axis = a.axis[j];
    if (tk < a.tokens && axis >= 0) {
      const int64_t tb = tk / a.rows;
      w = turn(a.pos[tb * a.p_sb + (tk - tb * a.rows) * a.p_st + axis], a.freq[j], a.inverse);
    }
    s_turn[r][j] = w;
  }
  __syncthreads();
  float2 w[PER];   // HALVES: of pairs ch ..; else of each chunk's
#pragma unroll
  for (int j = 0; j < PER; ++j)
    w[j] = s_turn[row][HALVES ? ch + j : ch / 2 + j % (N / 2) + j / (N / 2) * (H2 / 2)];

  for (; h < h_end; h += U * SLOTS) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int hu = h + u * SLOTS;
      if (hu >= h_end) continue;
      float x[E][N];
#pragma unroll
      for (int e = 0; e < E; ++e) v[u][e].get(x[e]);
      if constexpr (HALVES) {
#pragma unroll
        for (int j = 0; j < N; ++j) turn_pair(x[0][j], x[1][j], w[j]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int j = 0; j < N / 2; ++j) turn_pair(x[e][2 * j], x[e][2 * j + 1], w[e * (N / 2) + j]);
      }
      const bool second = hu >= a.heads[0];
      char* o = a.y[second] + (second ? y1 + (hu - a.heads[0]) * a.y_sh[1] : y0 + hu * a.y_sh[0]) * SIZE;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[u][e].set(x[e]);
        v[u][e].store(o + e * H2 * SIZE);
      }
    }
    load(h + U * SLOTS);
  }
}

template <int D, bool F32>
hipError_t launch_d(const TurnArgs& a, int pairs, hipStream_t s) {
  const unsigned grid = (unsigned)((a.tokens + kRopeRows - 1) / kRopeRows * a.head_parts);
  if (pairs == SSBA_ROPE_HALVES)
    k_rope<D, F32, true><<<grid, 256, 0, s>>>(a);
  else
    k_rope<D, F32, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_turn(const TurnArgs& a, int head_dim, int dtype, int pairs, hipStream_t s) {
  if (head_dim == 64) return dtype == SSBA_DT_F32 ? launch_d<64, true>(a, pairs, s) : launch_d<64, false>(a, pairs, s);
  return dtype == SSBA_DT_F32 ? launch_d<128, true>(a, pairs, s) : launch_d<128, false>(a, pairs, s);
}

}  // namespace ssba
