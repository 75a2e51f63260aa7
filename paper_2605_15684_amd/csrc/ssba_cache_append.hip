// New keys and values into the pages of a cache (include/ssba_cache.h).
//
// One workgroup per (sequence, page it touches, kv head).  A thread holds 4
// tokens x 8 channels of K and the same of V, so that 16 (D 128) lanes read a
// row's 256 bytes at once.  The page's exponent is the maximum over its new
// tokens and what it had.  The codes of a page that is new as a whole are put
// together in the LDS in the page's byte order and leave in 16-byte stores,
// 1 KB a wave; other pages get their few bytes directly.
// The sum of a page's codes is exact in fp32 (at most 64 codes of at most 448
// in steps of 2^-9: 24 bits), in any order.
// Bound by bytes, new rows read once and one byte a value written: four prompts
// of 5 to 8 thousand tokens, 8 heads, D 128 bf16 (109 MB) take 24 us, 4.5 TB/s;
// one token of each of 8 sequences takes 6 us, its chain of dependent loads.
#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>

#include "ssba_cache_common.h"

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

// Four values of at most 448 as e4m3, to nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ __forceinline__ void values_of(uint32_t w, float (&x)[4]) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}

// Eight consecutive values as they are in memory, and as numbers.
template <bool F32>
struct Raw {
  u32x4 w[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* base, int64_t off) {
    if (F32) {
      const float* p = static_cast<const float*>(base) + off;
      w[0] = *reinterpret_cast<const u32x4a4*>(p);
      w[F32 ? 1 : 0] = *reinterpret_cast<const u32x4a4*>(p + 4);
    } else {
      w[0] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + off);
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (F32) {
        x[e] = __uint_as_float(w[0][e]);
        x[4 + e] = __uint_as_float(w[F32 ? 1 : 0][e]);
      } else {
        x[2 * e] = __uint_as_float(w[0][e] << 16);
        x[2 * e + 1] = __uint_as_float(w[0][e] & 0xffff0000u);
      }
    }
  }
};

template <int D, bool F32>
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  constexpr int NCH = D / 8;
  __shared__ uint32_t s_top[2];
  __shared__ float s_sum[4][D];
  __shared__ u32x4 s_page[2][64 * D / 16];   // the codes of a new page
  const int page = 1 << a.c.page_log2;
  unsigned id = blockIdx.x;
  const int h = id % a.c.kv_heads;
  id /= a.c.kv_heads;
  const int slot = id % a.slots;
  const int seq = id / a.slots;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int start = sv.start;
  if (sv.n == 0 || start < 0) return;
  const int lp = (start >> a.c.page_log2) + slot;
  if (lp > (sv.len - 1) >> a.c.page_log2) return;
  const int p0 = lp << a.c.page_log2;
  const int phys = a.b.table[(int64_t)seq * a.b.max_pages + lp];
  if (phys < 0 || phys >= a.c.pages) return;

  const int units = page * NCH / 4;            // threads with a part of the page
  const bool active = (int)threadIdx.x < units;
  const int ch8 = threadIdx.x % NCH, tq = threadIdx.x / NCH;   // channels 8 ch8 .., tokens 4 tq ..
  const bool complete = p0 + page <= sv.len;
  const bool has_old = p0 < start;
  float* scale = a.c.scale + ((int64_t)phys * a.c.kv_heads + h) * 2;
  uint32_t was[2] = {0, 0};
  if (has_old) {
    was[0] = __float_as_uint(scale[0]);
    was[1] = __float_as_uint(scale[1]);
  }
  if (threadIdx.x < 2) s_top[threadIdx.x] = 0;

  // Every thread loads four rows at once; where it has none of the page's new
  // ones, the sequence's first new row stands in (its values count for nothing).
  bool fresh[4], old[4];
  Raw<F32> raw[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pos = p0 + 4 * tq + i;
    fresh[i] = active && pos >= start && pos < sv.len;
    old[i] = active && pos < start;
    const int64_t off = (int64_t)(sv.begin + (fresh[i] ? pos - start : 0)) * a.st + (int64_t)h * a.sh + ch8 * 8;
    raw[0][i].load(a.k, off);
    raw[1][i].load(a.v, off);
  }
  float x[2][4][8];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv)
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[kv][i].get(x[kv][i]);
  __syncthreads();   // every thread has the old scales before they are replaced
  // The largest magnitude; fmaxf passes over NaN.
  float top[2] = {0.f, 0.f};
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (fresh[i]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top[kv] = fmaxf(top[kv], fabsf(x[kv][i][e]));
      }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top[kv] = fmaxf(top[kv], __shfl_xor(top[kv], off));
    if ((threadIdx.x & 63) == 0) atomicMax(&s_top[kv], __float_as_uint(top[kv]));
  }
  __syncthreads();
  const bool infinite[2] = {s_top[0] == 0x7f800000u, s_top[1] == 0x7f800000u};
  if (infinite[0] || infinite[1]) {   // rare: once more over the finite ones
    __syncthreads();
    if (threadIdx.x < 2) s_top[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (fresh[i]) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t b = __float_as_uint(x[kv][i][e]) & 0x7fffffffu;
            t = max(t, b < 0x7f800000u ? b : 0u);
          }
        }
      if (t) atomicMax(&s_top[kv], t);
    }
    __syncthreads();
  }

  int e[2];
  float inv[2], restate[2];
  bool grows[2];   // older codes change: the scale is not what it was
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    e[kv] = exponent_of(s_top[kv]);
    restate[kv] = 1.f;
    if (has_old) {
      // The smallest power of two that reaches the old scale, which need not be one itself.
      const int up = (was[kv] & 0x7fffffu) ? 1 : 0;
      e[kv] = max(e[kv], min(max((int)((was[kv] >> 23) & 0xff) - 127 + up, kMinExp), kMaxExp));
      restate[kv] = __uint_as_float(was[kv]) * pow2(-e[kv]);
    }
    grows[kv] = restate[kv] != 1.f;
    inv[kv] = pow2(-e[kv]);
    if (threadIdx.x == 0) scale[kv] = pow2(e[kv]);
    if (infinite[kv]) {   // infinities take the largest code: scaled here, once and for all
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float y = x[kv][i][c] * inv[kv];
          x[kv][i][c] = fabsf(y) > 448.f ? copysignf(448.f, y) : y;
        }
      inv[kv] = 1.f;
    }
  }
  const int64_t image = (int64_t)phys * a.c.page_bytes + (int64_t)h * page * D;
  // Bytes of this thread's first token in the page: 8 of K (then 16 on per
  // token), a word of V per channel.
  const int block = (tq >> 2) * 16 * D + (ch8 >> 3) * 1024;
  const int k_at = block + (ch8 >> 1 & 3) * 256 + (tq & 3) * 64 + (ch8 & 1) * 8;
  const int v_at = block + (tq & 3) * 256 + (ch8 & 1) * 128 + (ch8 >> 1 & 3) * 4;
  float sum[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) sum[c] = 0.f;

  if (complete && !has_old) {
    // The whole page is new.
    if (active) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float(&y)[8] = x[0][i];
        const float f = inv[0];
        const uint32_t w0 = codes_of(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
        const uint32_t w1 = codes_of(y[4] * f, y[5] * f, y[6] * f, y[7] * f);
        *reinterpret_cast<uint2*>(reinterpret_cast<char*>(s_page[0]) + k_at + 16 * i) = make_uint2(w0, w1);
        float z[4];
        values_of(w0, z);
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += z[c];
        values_of(w1, z);
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[4 + c] += z[c];
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float f = inv[1];
        *reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(s_page[1]) + v_at + 16 * c) =
            codes_of(x[1][0][c] * f, x[1][1][c] * f, x[1][2][c] * f, x[1][3][c] * f);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < page * D / 16; i += blockDim.x) {
      *reinterpret_cast<u32x4*>(a.c.k + image + 16 * i) = s_page[0][i];
      *reinterpret_cast<u32x4*>(a.c.v + image + 16 * i) = s_page[1][i];
    }
  } else if (active) {
    uint8_t* kp = a.c.k + image + k_at;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[2] = {0, 0};   // stays 0 for what is neither read nor new: those count for nothing below
      const bool read = old[i] && (grows[0] || complete);
      if (read) {
        const uint2 c = *reinterpret_cast<const uint2*>(kp + 16 * i);
        w[0] = c.x;
        w[1] = c.y;
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float y[4];
        if (fresh[i]) {
          const float f = inv[0];
          w[q] = codes_of(x[0][i][4 * q] * f, x[0][i][4 * q + 1] * f, x[0][i][4 * q + 2] * f, x[0][i][4 * q + 3] * f);
        } else if (read && grows[0]) {
          values_of(w[q], y);
          w[q] = codes_of(y[0] * restate[0], y[1] * restate[0], y[2] * restate[0], y[3] * restate[0]);
        }
        values_of(w[q], y);
#pragma unroll
        for (int z = 0; z < 4; ++z) sum[4 * q + z] += y[z];
      }
      if (fresh[i] || (old[i] && grows[0])) *reinterpret_cast<uint2*>(kp + 16 * i) = make_uint2(w[0], w[1]);
    }
    uint8_t* vp = a.c.v + image + v_at;
    bool write[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) write[i] = fresh[i] || (old[i] && grows[1]);
    const bool all = write[0] && write[1] && write[2] && write[3];
    const bool any_old = grows[1] && (old[0] || old[1] || old[2] || old[3]);
    if (write[0] || write[1] || write[2] || write[3]) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        if (any_old) values_of(*reinterpret_cast<const uint32_t*>(vp + c * 16), y);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = fresh[i] ? x[1][i][c] * inv[1] : y[i] * restate[1];
        const uint32_t w = codes_of(y[0], y[1], y[2], y[3]);
        if (all) {
          *reinterpret_cast<uint32_t*>(vp + c * 16) = w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (write[i]) vp[c * 16 + i] = (uint8_t)(w >> (8 * i));
        }
      }
    }
  }

  if (!complete) return;
  // Sum of the codes over the page's tokens: the threads of a channel block
  // are NCH apart.
#pragma unroll
  for (int c = 0; c < 8; ++c)
#pragma unroll
    for (int off = NCH; off < 64; off <<= 1) sum[c] += __shfl_xor(sum[c], off);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane < NCH) {
#pragma unroll
    for (int c = 0; c < 8; ++c) s_sum[wave][lane * 8 + c] = sum[c];
  }
  __syncthreads();
  const float f = pow2(e[0]) / (float)page;
  __hip_bfloat16* mean = reinterpret_cast<__hip_bfloat16*>(a.c.kmean) + ((int64_t)phys * a.c.kv_heads + h) * D;
  for (int c = threadIdx.x; c < D; c += blockDim.x) {
    float t = s_sum[0][c];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) t += s_sum[w][c];
    mean[c] = __float2bfloat16(t * f);
  }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t s) {
  const int64_t groups = (int64_t)a.b.seqs * a.slots * a.c.kv_heads;
  const int threads = max(64, (a.c.head_dim << a.c.page_log2) / 32);
  const bool f32 = dtype == SSBA_DT_F32;
  auto go = [&](auto k) { k<<<(unsigned)groups, threads, 0, s>>>(a); };
  if (a.c.head_dim == 64) f32 ? go(k_cache_append<64, true>) : go(k_cache_append<64, false>);
  else f32 ? go(k_cache_append<128, true>) : go(k_cache_append<128, false>);
  return hipGetLastError();
}

}  // namespace ssba
