// Block selection for single queries (include/ssba_cache.h): a score of every
// page between the ones always kept, then the largest of them per token and kv
// head.
//
// Scores are in 64 bits, where a sum of products of bf16 numbers over at most
// 128 channels has few roundings or none: lists are those of the exact scores
// except where two of these differ by less than about 1e-16 of their terms.
// Within a list every page's sum is formed in the same order, so equal pages
// have equal scores.  Ranking is on 64-bit keys whose order is that of the
// scores (rank_key).
//
//   k_select_row     one (token, kv head) per workgroup, tables of at most 1152
//                    pages: scores into the LDS, one wave ranks them.  Bound by
//                    the pooled keys, 2 D bytes a page.
//   k_select_tile    16 tokens of a sequence per workgroup: a page's pooled key
//                    serves them all, on v_mfma_f64_16x16x4_f64.  Scores into
//                    the LDS (at most 1152 pages), or to the scratch.
//   k_select_scores, k_select_top(_waves)   longer tables: a row's pages are
//                    shared out over workgroups, then one workgroup (where
//                    there are many rows, one wave) ranks the row.
// Measured, D 128: 52 tokens x 4 heads x 130 to 256 pages 9.4 us (row); 1024
// tokens x 8 heads x 384 pages, D 64, 21.4 us (tile; the ranking 7, the matrix
// instructions 5); one token x 4 heads x 4096 pages 5.0 + 8.5 us.
#include <hip/hip_runtime.h>

#include <cstring>

#include "ssba_cache_common.h"
#include "ssba_common.h"

namespace ssba {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef double doublex4 __attribute__((ext_vector_type(4)));

// The pages a token can choose from: [first, first + middle) are scored.
struct Range {
  int total, middle;
};

__device__ __forceinline__ Range range_of(const SelectArgs& a, const SeqView& sv, int tok) {
  const int seen = a.causal ? min(sv.start + tok + 1, sv.len) : sv.len;
  Range r;
  r.total = seen > 0 ? ((seen - 1) >> a.c.page_log2) + 1 : 0;
  r.middle = r.total > a.keep ? r.total - a.first - a.last : 0;
  return r;
}

// Sum over the group's query heads, in order, of N channels from `ch` of a row.
template <bool F32, int N>
__device__ __forceinline__ void q_sum(const SelectArgs& a, int row, int h, int ch, double (&q)[N]) {
  constexpr int W = F32 ? N : N / 2;   // words
#pragma unroll
  for (int c = 0; c < N; ++c) q[c] = 0.0;
  const int64_t at = (int64_t)row * a.st + (int64_t)h * a.group * a.sh + ch;
#pragma unroll 2
  for (int g = 0; g < a.group; ++g) {
    uint32_t w[W];
    if (F32) {
      std::memcpy(w, __builtin_assume_aligned(static_cast<const float*>(a.q) + at + g * a.sh, 4), 4 * W);
#pragma unroll
      for (int c = 0; c < W; ++c) q[c] += (double)__uint_as_float(w[c]);
    } else {
      std::memcpy(w, __builtin_assume_aligned(static_cast<const uint16_t*>(a.q) + at + g * a.sh, 2 * N), 4 * W);
#pragma unroll
      for (int c = 0; c < W; ++c) {
        q[2 * c < N ? 2 * c : 0] += (double)__uint_as_float(w[c] << 16);
        q[2 * c + 1 < N ? 2 * c + 1 : 0] += (double)__uint_as_float(w[c] & 0xffff0000u);
      }
    }
  }
}

__device__ __forceinline__ bool page_of(const SelectArgs& a, const int32_t* table, int j, int* p) {
  *p = table[j];
  const bool there = *p >= 0 && *p < a.c.pages;
  if (!there) *p = 0;
  return there;
}

// What every list begins and ends with; false if that is all of it.  `t` of
// `n` threads.
__device__ __forceinline__ bool list_ends(const SelectArgs& a, const Range& r, int32_t* list, int t, int n) {
  const int count = min(r.total, a.keep);
  if (t == 0) list[0] = count;
  if (r.middle == 0) {
    for (int i = t; i < a.keep; i += n) list[1 + i] = i < count ? i : -1;
    return false;
  }
  for (int i = t; i < a.first; i += n) list[1 + i] = i;
  for (int i = t; i < a.last; i += n) list[1 + a.keep - a.last + i] = r.total - a.last + i;
  return a.keep - a.first - a.last > 0;
}

// Maximum over the wave, on the VALU (row shifts within 16 lanes, then
// broadcasts of a row's last lane); lanes whose source is not there keep 0.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));   // row_shr 1
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));   // row_bcast 15
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));   // row_bcast 31
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// One wave: the pages of the `need` largest of n <= 64 C keys, ascending, to
// out (page = base + index).  n > need.  The threshold is found bit by bit,
// first among the keys' high words, then among the low words of those equal
// there; the search ends where exactly as many keys lie above as are needed.
// If enough scores are within 1/8 of the largest, the search starts at the
// first bit in which keys of that range differ.
template <int C>
__device__ __forceinline__ void wave_top(const uint64_t* keys, int n, int need, int base, int32_t* out, int lane) {
  uint32_t hi[C], lo[C];
  uint32_t most = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint64_t k = c * 64 + lane < n ? keys[c * 64 + lane] : 0;
    hi[c] = (uint32_t)(k >> 32);
    lo[c] = (uint32_t)k;
    most = max(most, hi[c]);
  }
  most = wave_max(most);
  uint32_t th = 0, tl = 0;
  int b = 31;
  constexpr uint32_t kEighth = 3u << 20;   // of the exponent, in a key's high word
  if (most >= 0x80000000u + kEighth) {
    const uint32_t from = most - kEighth;
    int cnt = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) cnt += __popcll(__builtin_amdgcn_ballot_w64(hi[c] >= from));
    if (cnt >= need) {   // from <= threshold <= most
      b = 31 - __builtin_clz(from ^ most);
      th = most & ~((2u << b) - 1u);
    }
  }
  int left = need;       // places for keys whose high word is th
  bool low = true;       // the low words decide
  for (; b >= 0; --b) {
    const uint32_t cand = th | (1u << b);
    int cnt = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) cnt += __popcll(__builtin_amdgcn_ballot_w64(hi[c] >= cand));
    if (cnt >= need) {
      th = cand;
      if (cnt == need) {
        low = false;
        break;
      }
    }
  }
  if (low) {
#pragma unroll
    for (int c = 0; c < C; ++c) left -= __popcll(__builtin_amdgcn_ballot_w64(hi[c] > th));
    for (int bl = 31; bl >= 0; --bl) {
      const uint32_t cand = tl | (1u << bl);
      int cnt = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) cnt += __popcll(__builtin_amdgcn_ballot_w64(hi[c] == th && lo[c] >= cand));
      if (cnt >= left) {
        tl = cand;
        if (cnt == left) break;
      }
    }
  }
  // Above the threshold, and of those at it the first ones.
  int at_rest = need, at = 0;
#pragma unroll
  for (int c = 0; c < C; ++c)
    at_rest -= __popcll(__builtin_amdgcn_ballot_w64(hi[c] > th || (low && hi[c] == th && lo[c] > tl)));
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const bool in = c * 64 + lane < n;
    const bool gt = hi[c] > th || (low && hi[c] == th && lo[c] > tl);
    const bool eq = in && hi[c] == th && (!low || lo[c] == tl);
    const uint64_t meq = __builtin_amdgcn_ballot_w64(eq);
    const bool take = gt || (eq && __popcll(meq & below) < at_rest);
    const uint64_t mt = __builtin_amdgcn_ballot_w64(take);
    if (take) out[at + __popcll(mt & below)] = base + c * 64 + lane;
    at += __popcll(mt);
    at_rest -= min(at_rest, __popcll(meq));
  }
}

// n <= CAP
template <int CAP>
__device__ __forceinline__ void wave_top_any(const uint64_t* keys, int n, int need, int base, int32_t* out, int lane) {
  if (n <= 128) wave_top<2>(keys, n, need, base, out, lane);
  else if (n <= 256) wave_top<4>(keys, n, need, base, out, lane);
  else if (CAP > 256 && n <= 384) wave_top<6>(keys, n, need, base, out, lane);
  else if (CAP > 256 && n <= 512) wave_top<8>(keys, n, need, base, out, lane);
  else if (CAP > 512) wave_top<kSelectInLds / 64>(keys, n, need, base, out, lane);
}

// Ranking keys of pages j0, j0 + step, ... below `end` by one row's queries: D / 8 lanes to a page.
template <int D, int UNROLL>
__device__ __forceinline__ void score_pages(const SelectArgs& a, const int32_t* table, int h, const double (&q)[8],
                                            int sub, int j0, int step, int end, uint64_t* keys) {
  constexpr int LPP = D / 8;
  for (int j = j0; j < end; j += step * UNROLL) {
    u32x4 w[UNROLL];
    bool there[UNROLL];
    int p[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) there[u] = page_of(a, table, min(j + u * step, end - 1), &p[u]);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
      w[u] = *reinterpret_cast<const u32x4*>(a.c.kmean + ((int64_t)p[u] * a.c.kv_heads + h) * D + sub * 8);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      double s = 0.0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s += q[2 * c] * (double)__uint_as_float(w[u][c] << 16);
        s += q[2 * c + 1] * (double)__uint_as_float(w[u][c] & 0xffff0000u);
      }
#pragma unroll
      for (int off = 1; off < LPP; off <<= 1) s += __shfl_xor(s, off);
      if (sub == 0 && j + u * step < end) keys[j + u * step] = there[u] ? rank_key(s) : 0;
    }
  }
}

constexpr int kRowThreads = 512;

template <int D, bool F32>
__global__ __launch_bounds__(kRowThreads) void k_select_row(SelectArgs a) {
  constexpr int LPP = D / 8;
  __shared__ uint64_t s_keys[kSelectInLds];
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x / a.c.kv_heads, h = blockIdx.x % a.c.kv_heads;
  double q[8];   // its loads go out before those that find the row's sequence
  q_sum<F32, 8>(a, row, h, lane % LPP * 8, q);
  int seq;
  SeqView sv;
  if (!seq_of_row(a.b, a.c.page_log2, row, lane, &seq, &sv)) return;
  const int tok = row - sv.begin;
  const Range r = range_of(a, sv, tok);
  int32_t* list = a.lists + ((int64_t)row * a.c.kv_heads + h) * (1 + a.keep);
  if (!list_ends(a, r, list, threadIdx.x, kRowThreads)) return;
  const int32_t* table = a.b.table + (int64_t)seq * a.b.max_pages + a.first;
  score_pages<D, 4>(a, table, h, q, lane % LPP, threadIdx.x / LPP, kRowThreads / LPP, r.middle, s_keys);
  __syncthreads();
  if (threadIdx.x < 64)
    wave_top_any<kSelectInLds>(s_keys, r.middle, a.keep - a.first - a.last, a.first, list + 1 + a.first, lane);
}

// 16 tokens x all their pages.  A: the tokens' query sums, channels
// g D/4 .. of lane group g; B: 16 pages' pooled keys, the same channels; a
// lane gets the scores of tokens 4 i + g with page lane % 16.
template <int D, bool F32, int CAP, bool LDS>
__global__ __launch_bounds__(kRowThreads) void k_select_tile(SelectArgs a) {
  constexpr int CH = D / 4, WAVES = kRowThreads / 64, QL = D + 2;   // QL: 16 rows in 16 banks
  __shared__ alignas(16) uint64_t s_keys[16 * (LDS ? CAP : QL)];
  static_assert(!LDS || CAP >= QL, "");
  const int lane = threadIdx.x & 63, n16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned id = blockIdx.x;
  const int tile = id % a.tiles;
  id /= a.tiles;
  const int h = id % a.c.kv_heads, seq = id / a.c.kv_heads;
  const SeqView sv = seq_view(a.b, a.c.page_log2, seq);
  const int tok0 = tile * 16, last = min(min(sv.n, a.b.max_new), tok0 + 16) - 1;
  if (last < tok0) return;
  const int most = range_of(a, sv, last).middle;   // later tokens see more
  if (most > 0 && a.keep > a.first + a.last) {
    // The tokens' query sums through the LDS, a share of them by each thread: additions of 64 bits are slow (512
    // tokens x 4 heads, D 128, 16 query heads each: 15.5 us, every wave for itself 26).
    {
      constexpr int PT = D / 32;   // channels of a thread
      const int t = threadIdx.x / 32, c0 = threadIdx.x % 32 * PT;
      double sum[PT];
      q_sum<F32, PT>(a, sv.begin + min(tok0 + t, last), h, c0, sum);
#pragma unroll
      for (int c = 0; c < PT; ++c) s_keys[t * QL + c0 + c] = (uint64_t)__double_as_longlong(sum[c]);
    }
    __syncthreads();
    double q[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) q[c] = __longlong_as_double((long long)s_keys[n16 * QL + g * CH + c]);
    if (LDS) __syncthreads();
    const int32_t* table = a.b.table + (int64_t)seq * a.b.max_pages + a.first;
    int middle[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) middle[i] = tok0 + 4 * i + g <= last ? range_of(a, sv, tok0 + 4 * i + g).middle : 0;
    for (int j0 = (wave * gridDim.y + blockIdx.y) * 16; j0 < most; j0 += WAVES * 16 * gridDim.y) {
      int p;
      const bool there = page_of(a, table, min(j0 + n16, most - 1), &p);
      const uint16_t* mean = a.c.kmean + ((int64_t)p * a.c.kv_heads + h) * D + g * CH;
      u32x4 w[CH / 8];
#pragma unroll
      for (int c = 0; c < CH / 8; ++c) w[c] = *reinterpret_cast<const u32x4*>(mean + c * 8);
      doublex4 s = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const uint32_t x = w[c / 8][(c % 8) / 2];
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(q[c], (double)__uint_as_float(c & 1 ? x & 0xffff0000u : x << 16), s, 0,
                                                 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (j0 + n16 >= middle[i]) continue;
        const uint64_t key = there ? rank_key(s[i]) : 0;
        if (LDS) s_keys[(4 * i + g) * CAP + j0 + n16] = key;
        else a.keys[((int64_t)(sv.begin + tok0 + 4 * i + g) * a.c.kv_heads + h) * a.b.max_pages + j0 + n16] = key;
      }
    }
  }
  if (!LDS) return;
  __syncthreads();
  for (int t = wave; t <= last - tok0; t += WAVES) {
    const Range r = range_of(a, sv, tok0 + t);
    int32_t* list = a.lists + ((int64_t)(sv.begin + tok0 + t) * a.c.kv_heads + h) * (1 + a.keep);
    if (list_ends(a, r, list, lane, 64))
      wave_top_any<CAP>(&s_keys[t * CAP], r.middle, a.keep - a.first - a.last, a.first, list + 1 + a.first, lane);
  }
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void k_select_scores(SelectArgs a) {
  constexpr int LPP = D / 8;
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x / a.c.kv_heads, h = blockIdx.x % a.c.kv_heads;
  int seq;
  SeqView sv;
  if (!seq_of_row(a.b, a.c.page_log2, row, lane, &seq, &sv)) return;
  const int tok = row - sv.begin;
  const Range r = range_of(a, sv, tok);
  if ((int)blockIdx.y * kSelectPages >= r.middle) return;
  double q[8];
  q_sum<F32, 8>(a, row, h, lane % LPP * 8, q);
  const int32_t* table = a.b.table + (int64_t)seq * a.b.max_pages + a.first;
  uint64_t* keys = a.keys + ((int64_t)row * a.c.kv_heads + h) * a.b.max_pages;
  for (int j0 = blockIdx.y * kSelectPages; j0 < r.middle; j0 += gridDim.y * kSelectPages)
    score_pages<D, kSelectPages * LPP / 256>(a, table, h, q, lane % LPP, j0 + threadIdx.x / LPP, 256 / LPP,
                                             min(j0 + kSelectPages, r.middle), keys);
}

// One workgroup per (row, kv head): the `need` largest keys by radix, 8 bits a
// pass, then their pages in ascending order.  Digits are of the keys' distance
// from the largest high word: where enough scores are within 2^-16 of the
// largest, whose distances share their first byte, that pass is left out.  A
// pass has one barrier: every wave looks through the bins, of which there are
// three sets, one counted, one looked through, one cleared.
// 4 rows of 4096 pages: 8.5 us (16 waves: few barriers, long chains).
constexpr int kTopThreads = 1024, kTopWaves = kTopThreads / 64, kTopRegs = 8;
constexpr int kTopKeys = kTopRegs * kTopThreads;

// Inclusive sum over the lanes up to each.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(x, off);
    if (lane >= off) x += o;
  }
  return x;
}

__global__ __launch_bounds__(kTopThreads) void k_select_top(SelectArgs a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x / a.c.kv_heads, h = blockIdx.x % a.c.kv_heads;
  int seq;
  SeqView sv;
  if (!seq_of_row(a.b, a.c.page_log2, row, lane, &seq, &sv)) return;
  const int tok = row - sv.begin;
  const Range r = range_of(a, sv, tok);
  int32_t* list = a.lists + ((int64_t)row * a.c.kv_heads + h) * (1 + a.keep);
  if (!list_ends(a, r, list, threadIdx.x, kTopThreads)) return;
  const int need = a.keep - a.first - a.last;   // < r.middle
  const uint64_t* keys = a.keys + ((int64_t)row * a.c.kv_heads + h) * a.b.max_pages;

  // The first kTopRegs keys of each thread stay in registers.
  uint64_t mine[kTopRegs];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < kTopRegs; ++i) {
    const int j = i * kTopThreads + threadIdx.x;
    mine[i] = j < r.middle ? keys[j] : 0;
    most = max(most, (uint32_t)(mine[i] >> 32));
  }
  for (int j = kTopKeys + threadIdx.x; j < r.middle; j += kTopThreads) most = max(most, (uint32_t)(keys[j] >> 32));
  __shared__ int s_hist[3][256];
  __shared__ uint32_t s_most[kTopWaves];
  __shared__ int s_wave[kTopRegs * kTopWaves];
  most = wave_max(most);
  if (lane == 0) s_most[wave] = most;
  if (threadIdx.x < 3 * 256) s_hist[threadIdx.x >> 8][threadIdx.x & 255] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kTopWaves; ++w) most = max(most, s_most[w]);
  const uint64_t top = (uint64_t)most << 32 | 0xffffffffu;
#pragma unroll
  for (int i = 0; i < kTopRegs; ++i) mine[i] = top - mine[i];   // distances: the smallest are wanted

  uint64_t prefix = 0;   // the threshold's high bits
  int left = need;       // places for distances that match the prefix
  int shift = 56, set = 0;
  // Distances share their high bytes, so lanes of a wave with the same digit add once.
  auto count = [&](uint64_t d, bool in) {
    const int digit = (int)(d >> shift) & 255;
    bool todo = in && (shift == 56 || (d >> (shift + 8)) == (prefix >> (shift + 8)));
#pragma unroll
    for (int turn = 0; turn < 2; ++turn) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(todo);
      if (!m) return;
      const int first = __builtin_ctzll(m);
      const bool same = todo && digit == __builtin_amdgcn_readlane(digit, first);
      const uint64_t ms = __builtin_amdgcn_ballot_w64(same);
      if (lane == first) atomicAdd(&s_hist[set][digit], __popcll(ms));
      if (same) todo = false;
    }
    if (todo) atomicAdd(&s_hist[set][digit], 1);
  };
  for (bool skip = true;;) {
    if (skip) shift = 48;   // distances whose first byte is 0
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i)
      if (i * kTopThreads < r.middle) count(mine[i], i * kTopThreads + (int)threadIdx.x < r.middle);
    for (int j0 = kTopKeys; j0 < r.middle; j0 += kTopThreads) {
      const int j = j0 + threadIdx.x;
      count(j < r.middle ? top - keys[j] : 0, j < r.middle);
    }
    __syncthreads();
    // The bin in which the `left`-th distance lies.
    int c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] = s_hist[set][4 * lane + i];
      sum += c[i];
    }
    const int third = set == 0 ? 2 : set - 1;   // counted two passes on
    if (threadIdx.x < 256) s_hist[third][threadIdx.x] = 0;
    set = set == 2 ? 0 : set + 1;
    const int incl = wave_scan(sum, lane);
    const uint64_t reach = __builtin_amdgcn_ballot_w64(incl >= left);
    if (!reach) {   // fewer than `need` have a first byte of 0
      skip = false;
      shift = 56;
      continue;
    }
    skip = false;
    int before = incl - sum, bin = 0, in_bin = 0, above = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before < left && before + c[i] >= left) {
        bin = 4 * lane + i;
        in_bin = c[i];
        above = before;
      }
      before += c[i];
    }
    const int at = __builtin_ctzll(reach);
    bin = __builtin_amdgcn_readlane(bin, at);
    in_bin = __builtin_amdgcn_readlane(in_bin, at);
    prefix |= (uint64_t)bin << shift;
    left -= __builtin_amdgcn_readlane(above, at);
    if (in_bin == left || shift == 0) break;   // the whole bin is taken
    shift -= 8;
  }

  // Taken: distances below the threshold's prefix, and of those equal to it the first `left`.
  const uint64_t t = prefix >> shift;
  int base = a.first, equal_before = 0;
  for (int c0 = 0; c0 < r.middle; c0 += kTopKeys) {
    if (c0) {
#pragma unroll
      for (int i = 0; i < kTopRegs; ++i) {
        const int j = c0 + i * kTopThreads + threadIdx.x;
        mine[i] = j < r.middle ? top - keys[j] : 0;
      }
      __syncthreads();
    }
    // Equal and nearer ones of each wave and turn, counted together (16 bits each).
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      const bool in = c0 + i * kTopThreads + (int)threadIdx.x < r.middle;
      const uint64_t d = mine[i] >> shift;
      const uint64_t meq = __builtin_amdgcn_ballot_w64(in && d == t), mlt = __builtin_amdgcn_ballot_w64(in && d < t);
      if (lane == 0) s_wave[i * kTopWaves + wave] = __popcll(meq) | (__popcll(mlt) << 16);
    }
    __syncthreads();
    const int e0 = s_wave[2 * lane], e1 = s_wave[2 * lane + 1];
    const int incl = wave_scan(e0 + e1, lane), total = __builtin_amdgcn_readlane(incl, 63);
    const int ahead = wave & 1 ? incl - e1 : incl - e0 - e1;   // of the lane's entry of this wave's parity
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      const int j = c0 + i * kTopThreads + threadIdx.x;
      const bool in = j < r.middle;
      const uint64_t d = mine[i] >> shift;
      const bool eq = in && d == t, lt = in && d < t;
      const uint64_t meq = __builtin_amdgcn_ballot_w64(eq), mlt = __builtin_amdgcn_ballot_w64(lt);
      const int before = __builtin_amdgcn_readlane(ahead, (i * kTopWaves + wave) >> 1) +
                         (__popcll(meq & below) | (__popcll(mlt & below) << 16));
      const int rank = equal_before + (before & 0xffff);
      // Taken ones in front: all nearer ones, and the equal ones that have a place.
      if (lt || (eq && rank < left))
        list[1 + base + (before >> 16) + min(rank, left) - min(equal_before, left)] = a.first + j;
    }
    base += (total >> 16) + min(equal_before + (total & 0xffff), left) - min(equal_before, left);
    equal_before += total & 0xffff;
  }
}

// Many rows of moderate length: a wave ranks a row of at most 64 C pages, its
// keys in registers.
template <int C>
__global__ __launch_bounds__(256) void k_select_top_waves(SelectArgs a) {
  const int lane = threadIdx.x & 63;
  const unsigned id = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = __builtin_amdgcn_readfirstlane(id / a.c.kv_heads);
  const int h = __builtin_amdgcn_readfirstlane(id % a.c.kv_heads);
  int seq;
  SeqView sv;
  if (row >= a.b.rows || !seq_of_row(a.b, a.c.page_log2, row, lane, &seq, &sv)) return;
  const Range r = range_of(a, sv, row - sv.begin);
  const int64_t at = (int64_t)row * a.c.kv_heads + h;
  int32_t* list = a.lists + at * (1 + a.keep);
  if (list_ends(a, r, list, lane, 64))
    wave_top<C>(a.keys + at * a.b.max_pages, r.middle, a.keep - a.first - a.last, a.first, list + 1 + a.first, lane);
}

template <int D, bool F32>
hipError_t launch(const SelectArgs& a, const SelectPlan& p, hipStream_t s) {
  const unsigned rows = (unsigned)a.b.rows * a.c.kv_heads;
  const unsigned tiles = (unsigned)a.b.seqs * a.c.kv_heads * a.tiles;
  switch (p.kind) {
    case kSelectRow:
      k_select_row<D, F32><<<rows, kRowThreads, 0, s>>>(a);
      break;
    case kSelectTile:
      if (a.b.max_pages <= 256) k_select_tile<D, F32, 256, true><<<tiles, kRowThreads, 0, s>>>(a);
      else if (a.b.max_pages <= 512) k_select_tile<D, F32, 512, true><<<tiles, kRowThreads, 0, s>>>(a);
      else k_select_tile<D, F32, kSelectInLds, true><<<tiles, kRowThreads, 0, s>>>(a);
      break;
    default: {
      if (p.scored) {
        if (p.kind == kSelectTileLong) k_select_tile<D, F32, 1, false><<<dim3(tiles, p.chunks), kRowThreads, 0, s>>>(a);
        else k_select_scores<D, F32><<<dim3(rows, p.chunks), 256, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      // 8192 rows of 1025 pages: a workgroup each 173 us, a wave each 36; 4 rows of 4096: 8.5 us in workgroups.
      if (rows >= 1024 && a.b.max_pages <= 2048) k_select_top_waves<32><<<(rows + 3) / 4, 256, 0, s>>>(a);
      else if (rows >= 1024 && a.b.max_pages <= 4096) k_select_top_waves<64><<<(rows + 3) / 4, 256, 0, s>>>(a);
      else k_select_top<<<rows, kTopThreads, 0, s>>>(a);
    }
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_select(const SelectArgs& a, const SelectPlan& p, int dtype, hipStream_t s) {
  const bool f32 = dtype == SSBA_DT_F32;
  if (a.c.head_dim == 64) return f32 ? launch<64, true>(a, p, s) : launch<64, false>(a, p, s);
  return f32 ? launch<128, true>(a, p, s) : launch<128, false>(a, p, s);
}

}  // namespace ssba
