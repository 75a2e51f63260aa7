// New keys and values into the pages of a cache (include/ssba_cache.h).
//
// One workgroup per (sequence, page it touches, kv head).  A thread holds 4
// tokens x 16 channels of K or of V: for K that is four 16-byte pieces of the
// page, for V 16 words of 4 tokens, so both are written from registers.  The
// page's exponent is the maximum over its new tokens and what it had; the
// codes' sum over a page is exact in fp32 (64 codes of at most 448 in steps of
// 2^-9: 24 bits), in any order.
#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>

#include "ssba_cache.h"

namespace ssba {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kMinExp = -64, kMaxExp = 120;   // what finite fp32 values need

// Smallest e >= kMinExp with |x| <= 448 * 2^e for the |x| of these fp32 bits
// (finite): 448 = 1.75 * 2^8.
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  const int k = (int)(bits >> 23) - 127;
  return max(k - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), kMinExp);
}

__device__ __forceinline__ float pow2(int e) {   // e <= 127; below -126 too small to matter
  return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

__device__ __forceinline__ float saturate(float x) {   // NaN stays
  return fabsf(x) > 448.f ? copysignf(448.f, x) : x;
}

// Four values as e4m3, to nearest even.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(saturate(a), saturate(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(saturate(c), saturate(d), w, true);
}

__device__ __forceinline__ void values_of(uint32_t w, float (&x)[4]) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

template <bool F32>
__device__ __forceinline__ void load16(const void* base, int64_t off, float (&x)[16]) {
  if (F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4a4*>(static_cast<const float*>(base) + off + 4 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = __uint_as_float(w[e]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + off + 8 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[8 * i + 2 * e] = __uint_as_float(w[e] << 16);
        x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    }
  }
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  constexpr int NCH = D / 16;
  const int page = 1 << a.c.page_log2;
  unsigned id = blockIdx.x;
  const int h = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int slot = id % a.slots;
  const int seq = id / a.slots;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int start = sv.len - sv.n;
  if (sv.n == 0 || start < 0) return;
  const int lp = (start >> a.c.page_log2) + slot;
  const int p0 = lp << a.c.page_log2;
  if (p0 >= sv.len) return;
  const int phys = a.b.table[(int64_t)seq * a.b.max_pages + lp];
  if (phys < 0 || phys >= a.c.pages) return;

  const int units = page * D / 64;             // threads of K, and of V
  const int which = threadIdx.x / units;       // 0: K, 1: V, above: idle
  const int u = threadIdx.x - which * units;
  const int ch16 = u % NCH, tq = u / NCH;      // channels 16 ch16 .., tokens 4 tq ..
  const bool active = which < 2;
  const bool complete = p0 + page <= sv.len;
  const bool has_old = p0 < start;

  __shared__ uint32_t s_top[2];
  __shared__ float s_sum[2][D];
  if (threadIdx.x < 2) s_top[threadIdx.x] = 0;
  __syncthreads();

  float x[4][16];
  uint32_t top = 0;
  bool fresh[4], old[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pos = p0 + 4 * tq + i;
    fresh[i] = active && pos >= start && pos < sv.len;
    old[i] = active && pos < start;
    if (fresh[i]) {
      const int64_t off = (int64_t)(sv.begin + pos - start) * a.st + (int64_t)h * a.sh + ch16 * 16;
      load16<F32>(which ? a.v : a.k, off, x[i]);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t b = __float_as_uint(x[i][e]) & 0x7fffffffu;
        top = max(top, b < 0x7f800000u ? b : 0u);
      }
    }
  }
  if (top) atomicMax(&s_top[which & 1], top);
  __syncthreads();

  const int kv = which & 1;
  float* scale = a.c.scale + ((int64_t)phys * a.c.kv_heads + h) * 2;
  int e = exponent_of(s_top[kv]), e0 = e;
  if (has_old) {
    e0 = min(max((int)((__float_as_uint(scale[kv]) >> 23) & 0xff) - 127, kMinExp), kMaxExp);
    e = max(e, e0);
  }
  __syncthreads();   // every thread has the old scale before it is replaced
  if (active && u == 0) scale[kv] = pow2(e);

  const float inv = pow2(-e), restate = pow2(e0 - e);
  const bool grows = has_old && e > e0;
  uint8_t* base = (kv ? a.c.v : a.c.k) + (int64_t)phys * a.c.page_bytes + (int64_t)h * page * D +
                  (tq >> 2) * 16 * D + (ch16 >> 2) * 1024;
  float sum[16];
#pragma unroll
  for (int c = 0; c < 16; ++c) sum[c] = 0.f;

  if (active && kv == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint8_t* at = base + (ch16 & 3) * 256 + ((tq & 3) * 4 + i) * 16;
      u32x4 w = {0, 0, 0, 0};
      const bool read = old[i] && (grows || complete);
      if (read) w = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float y[4];
        if (fresh[i]) {
          w[q] = codes_of(x[i][4 * q] * inv, x[i][4 * q + 1] * inv, x[i][4 * q + 2] * inv, x[i][4 * q + 3] * inv);
        } else if (read && grows) {
          values_of(w[q], y);
          w[q] = codes_of(y[0] * restate, y[1] * restate, y[2] * restate, y[3] * restate);
        }
        values_of(w[q], y);   // 0 where neither: not complete, or no such token
#pragma unroll
        for (int z = 0; z < 4; ++z) sum[4 * q + z] += y[z];
      }
      if (fresh[i] || (old[i] && grows)) *reinterpret_cast<u32x4*>(at) = w;
    }
  } else if (active) {
    uint8_t* at = base + (tq & 3) * 256 + (ch16 & 3) * 4;
    bool write[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) write[i] = fresh[i] || (old[i] && grows);
    const bool all = write[0] && write[1] && write[2] && write[3];
    const bool any_old = grows && (old[0] || old[1] || old[2] || old[3]);
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      float y[4] = {0.f, 0.f, 0.f, 0.f};
      if (any_old) values_of(*reinterpret_cast<const uint32_t*>(at + c * 16), y);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = fresh[i] ? x[i][c] * inv : y[i] * restate;
      const uint32_t w = codes_of(y[0], y[1], y[2], y[3]);
      if (all) {
        *reinterpret_cast<uint32_t*>(at + c * 16) = w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (write[i]) at[c * 16 + i] = (uint8_t)(w >> (8 * i));
      }
    }
  }

  if (!complete) return;
  // Sum of the codes over the page's tokens: the K threads of a channel block
  // are NCH apart.
#pragma unroll
  for (int c = 0; c < 16; ++c)
    for (int off = NCH; off < min(units, 64); off <<= 1) sum[c] += __shfl_xor(sum[c], off);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (active && kv == 0 && lane < NCH) {
#pragma unroll
    for (int c = 0; c < 16; ++c) s_sum[wave][lane * 16 + c] = sum[c];
  }
  __syncthreads();
  if (active && kv == 0) {
    const float f = pow2(e) / (float)page;
    __hip_bfloat16* mean = reinterpret_cast<__hip_bfloat16*>(a.c.kmean) + ((int64_t)phys * a.c.kv_heads + h) * D;
    for (int c = u; c < D; c += units)
      mean[c] = __float2bfloat16((units > 64 ? s_sum[0][c] + s_sum[1][c] : s_sum[0][c]) * f);
  }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t s) {
  const int64_t groups = (int64_t)a.b.seqs * a.slots * a.c.kv_heads;
  const int threads = max(64, (2 << a.c.page_log2) * a.c.head_dim / 64);
  const bool f32 = dtype == SSBA_DT_F32;
  auto go = [&](auto k) { k<<<(unsigned)groups, threads, 0, s>>>(a); };
  if (a.c.head_dim == 64) f32 ? go(k_cache_append<64, true>) : go(k_cache_append<64, false>);
  else f32 ? go(k_cache_append<128, true>) : go(k_cache_append<128, false>);
  return hipGetLastError();
}

}  // namespace ssba
