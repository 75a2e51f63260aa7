// Block selection for single queries (include/ssba_cache.h): a score of every
// page between the ones always kept, then the largest of them per token and kv
// head.
//
// Scores are in 64 bits: a sum of bf16 products over at most 128 channels has
// few roundings there, in a fixed order, so a list depends on nothing but the
// data.  k_select_scores is bound by the pooled keys it reads (2 D bytes a page
// and head); k_select_top ranks 64-bit keys whose order is that of the scores.
#include <hip/hip_runtime.h>

#include "ssba_cache.h"
#include "ssba_common.h"

namespace ssba {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The pages a token can choose from: [first, first + middle) are scored.
struct Range {
  int total, middle;
};

__device__ __forceinline__ Range range_of(const SelectArgs& a, const SeqView& sv, int tok) {
  const int seen = a.causal ? sv.len - sv.n + tok + 1 : sv.len;
  Range r;
  r.total = seen > 0 ? ((seen - 1) >> a.c.page_log2) + 1 : 0;
  r.middle = r.total > a.keep ? r.total - a.first - a.last : 0;
  return r;
}

template <bool F32>
__device__ __forceinline__ double q_at(const void* q, int64_t i) {
  if (F32) return (double)static_cast<const float*>(q)[i];
  return (double)__uint_as_float((uint32_t) static_cast<const uint16_t*>(q)[i] << 16);
}

// D / 8 lanes to a page, 8 channels each.
template <int D, bool F32>
__global__ __launch_bounds__(256) void k_select_scores(SelectArgs a) {
  constexpr int LPP = D / 8, PPW = 64 / LPP;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / a.c.kv_heads, h = blockIdx.x % a.c.kv_heads;
  const int seq = seq_of_row(a.b, row, lane);
  if (seq >= a.b.seqs) return;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int tok = row - sv.begin;
  if (tok < 0 || tok >= sv.n) return;
  const Range r = range_of(a, sv, tok);
  if ((int)blockIdx.y * kSelectPages >= r.middle) return;
  const int sub = lane % LPP;
  double q[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) q[c] = 0.0;
  for (int g = 0; g < a.group; ++g) {
    const int64_t at = (int64_t)row * a.st + (int64_t)(h * a.group + g) * a.sh + sub * 8;
#pragma unroll
    for (int c = 0; c < 8; ++c) q[c] += q_at<F32>(a.q, at + c);
  }
  const int32_t* table = a.b.table + (int64_t)seq * a.b.max_pages + a.first;
  uint64_t* keys = a.keys + ((int64_t)row * a.c.kv_heads + h) * a.b.max_pages;
  for (int j0 = blockIdx.y * kSelectPages; j0 < r.middle; j0 += gridDim.y * kSelectPages)
  for (int j = j0 + wave * PPW + lane / LPP, end = min(j0 + kSelectPages, r.middle); j < end; j += 4 * PPW) {
    const int p = table[j];
    const bool there = p >= 0 && p < a.c.pages;
    const uint16_t* mean = a.c.kmean + ((int64_t)(there ? p : 0) * a.c.kv_heads + h) * D + sub * 8;
    const u32x4 w = *reinterpret_cast<const u32x4*>(mean);
    double s = 0.0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      s += q[2 * c] * (double)__uint_as_float(w[c] << 16);
      s += q[2 * c + 1] * (double)__uint_as_float(w[c] & 0xffff0000u);
    }
#pragma unroll
    for (int off = 1; off < LPP; off <<= 1) s += __shfl_xor(s, off);
    if (sub == 0) keys[j] = there ? rank_key(s) : 0;
  }
}

// One workgroup per (row, kv head): the `need` largest keys by radix, 8 bits a
// pass, then their pages in ascending order.
__global__ __launch_bounds__(256) void k_select_top(SelectArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / a.c.kv_heads, h = blockIdx.x % a.c.kv_heads;
  const int seq = seq_of_row(a.b, row, lane);
  if (seq >= a.b.seqs) return;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int tok = row - sv.begin;
  if (tok < 0 || tok >= sv.n) return;
  const Range r = range_of(a, sv, tok);
  int32_t* list = a.lists + ((int64_t)row * a.c.kv_heads + h) * (1 + a.keep);
  const int count = min(r.total, a.keep);
  if (threadIdx.x == 0) list[0] = count;
  if (r.middle == 0) {
    for (int i = threadIdx.x; i < a.keep; i += 256) list[1 + i] = i < count ? i : -1;
    return;
  }
  for (int i = threadIdx.x; i < a.first; i += 256) list[1 + i] = i;
  for (int i = threadIdx.x; i < a.last; i += 256) list[1 + a.keep - a.last + i] = r.total - a.last + i;
  const int need = a.keep - a.first - a.last;
  if (need == 0) return;

  const uint64_t* keys = a.keys + ((int64_t)row * a.c.kv_heads + h) * a.b.max_pages;
  __shared__ int s_hist[256];
  __shared__ int s_bin, s_left, s_wave[4];
  uint64_t prefix = 0;   // the threshold's high bits
  int left = need;       // places for keys that match the prefix
  int shift = 64;
  while (shift > 0) {
    shift -= 8;
    s_hist[threadIdx.x] = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < r.middle; j += 256) {
      const uint64_t k = keys[j];
      if (shift == 56 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // Bins from the top: the one in which the `left`-th key lies.
    if (wave == 0) {
      int c[4], sum = 0;   // bins 255 - 4 lane - i
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = s_hist[255 - 4 * lane - i];
        sum += c[i];
      }
      int incl = sum;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(incl, off);
        if (lane >= off) incl += o;
      }
      int above = incl - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < left && above + c[i] >= left) {
          s_bin = 255 - 4 * lane - i;
          s_left = left - above;
        }
        above += c[i];
      }
    }
    __syncthreads();
    prefix |= (uint64_t)s_bin << shift;
    left = s_left;
    const int in_bin = s_hist[s_bin];
    __syncthreads();
    if (in_bin == left) break;   // the whole bin is taken
  }
  // Taken: keys above the threshold's prefix, and of those equal to it the first `left`.
  int base = a.first, equal_before = 0;
  for (int j0 = 0; j0 < r.middle; j0 += 256) {
    const int j = j0 + threadIdx.x;
    bool gt = false, eq = false;
    if (j < r.middle) {
      const uint64_t k = keys[j] >> shift, t = prefix >> shift;
      gt = k > t;
      eq = k == t;
    }
    const uint64_t meq = __builtin_amdgcn_ballot_w64(eq);
    if (lane == 0) s_wave[wave] = __popcll(meq);
    __syncthreads();
    int rank = equal_before + __popcll(meq & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) rank += s_wave[w];
    equal_before += s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3];
    __syncthreads();
    const bool take = gt || (eq && rank < left);
    const uint64_t mt = __builtin_amdgcn_ballot_w64(take);
    if (lane == 0) s_wave[wave] = __popcll(mt);
    __syncthreads();
    int at = base + __popcll(mt & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) at += s_wave[w];
    if (take) list[1 + at] = a.first + j;
    base += s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3];
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_cache_select(const SelectArgs& a, int dtype, hipStream_t s) {
  const unsigned items = (unsigned)a.b.rows * a.c.kv_heads;
  if (a.b.max_pages > a.keep) {
    const dim3 grid(items, (unsigned)a.chunks);
    const bool f32 = dtype == SSBA_DT_F32;
    auto go = [&](auto k) { k<<<grid, 256, 0, s>>>(a); };
    if (a.c.head_dim == 64) f32 ? go(k_select_scores<64, true>) : go(k_select_scores<64, false>);
    else f32 ? go(k_select_scores<128, true>) : go(k_select_scores<128, false>);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  k_select_top<<<items, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ssba
