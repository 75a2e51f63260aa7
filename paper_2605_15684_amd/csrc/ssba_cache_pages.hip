// Page bookkeeping of the cache (include/ssba_cache.h): one workgroup walks
// the small arrays (references, page table) and leaves a list of page copies;
// a second launch moves the pages of all layers.  The walk is bound by the
// latency of its steps (16 rows x 33 entries, 640 pages: fork 5.7 us, release
// 3.9, reserve 3.0; 64 rows x 257 entries: 18, 22, 17), the copy by HBM (100
// pages x 24 layers of 35 KB: 31 us, 5.6 TB/s read and written).
#include <hip/hip_runtime.h>

#include "ssba_cache_common.h"

namespace ssba {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSlices = 8;   // arrays are walked in up to 8 slices of kThreads elements at a time

// Sum of `n` over the threads in front of this one, and over all of them.  `s`
// is LDS of kWaves ints.
__device__ __forceinline__ int block_sum(int n, int* s, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = n;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(incl, off);
    if (lane >= off) incl += o;
  }
  __syncthreads();
  if (lane == 63) s[wave] = incl;
  __syncthreads();
  int before = incl - n, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? s[w] : 0;
    sum += s[w];
  }
  *total = sum;
  return before;
}

// Ranks of flags over `slices` slices of kThreads elements in order (element
// i kThreads + thread is slice i's): how many set ones are in front of each of
// this thread's, and their total.  `s` is LDS of kSlices * kWaves ints.
__device__ __forceinline__ void slice_ranks(const bool (&flag)[kSlices], int slices, int* s, int (&rank)[kSlices],
                                            int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t below = (1ull << lane) - 1;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    if (i >= slices) break;
    const uint64_t m = __builtin_amdgcn_ballot_w64(flag[i]);
    rank[i] = __popcll(m & below);
    if (lane == 0) s[i * kWaves + wave] = __popcll(m);
  }
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    if (i >= slices) break;
    rank[i] += sum;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s[i * kWaves + w];
      rank[i] += w < wave ? c : 0;
      sum += c;
    }
  }
  *total = sum;
}

__device__ __forceinline__ int held(const PagesArgs& a, int row) {
  return min(max(a.lens[row], 0), a.max_pages << a.page_log2);
}

__device__ __forceinline__ bool is_page(const PagesArgs& a, int p) { return p >= 0 && p < a.pages; }

// Read past the L1, which this kernel's own atomics do not update.
__device__ __forceinline__ int fresh(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The lowest `n` free pages, in order: fn(j, page) for j < n; returns how many
// of them there are.
template <typename F>
__device__ __forceinline__ int take_free(const PagesArgs& a, int n, int* s, F fn) {
  int got = 0;
  for (int p0 = 0; p0 < a.pages && got < n; p0 += kThreads * kSlices) {
    const int slices = min((a.pages - p0 + kThreads - 1) / kThreads, kSlices);
    bool free[kSlices];
    int rank[kSlices], total;
#pragma unroll
    for (int i = 0; i < kSlices; ++i) {
      const int p = p0 + i * kThreads + threadIdx.x;
      free[i] = p < a.pages && fresh(&a.refs[p]) == 0;
    }
    slice_ranks(free, slices, s, rank, &total);
#pragma unroll
    for (int i = 0; i < kSlices; ++i)
      if (free[i] && got + rank[i] < n) fn(got + rank[i], p0 + i * kThreads + (int)threadIdx.x);
    got += total;
  }
  return min(got, n);
}

// scratch: the entries that lack a page, then how many each row has.  A wave
// takes a row.
__global__ __launch_bounds__(kThreads) void k_pages_reserve(PagesArgs a) {
  __shared__ int s[kSlices * kWaves];
  int* miss = a.scratch;
  int* of_row = miss + (int64_t)a.rows * a.max_pages;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // fn(entry, how many lack a page in front of it in the row); the row's number of them
  auto lacking = [&](int row, auto fn) {
    const int need = (held(a, row) + (1 << a.page_log2) - 1) >> a.page_log2;
    const int32_t* t = a.table + (int64_t)row * a.max_pages;
    int n = 0;
    for (int i0 = 0; i0 < need; i0 += 256) {
      bool lacks[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 64 + lane;
        lacks[u] = i < need && !is_page(a, t[i]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint64_t m = __builtin_amdgcn_ballot_w64(lacks[u]);
        if (lacks[u]) fn(i0 + u * 64 + lane, n + __popcll(m & ((1ull << lane) - 1)));
        n += __popcll(m);
      }
    }
    return n;
  };
  for (int row = wave; row < a.rows; row += kWaves) {
    const int n = lacking(row, [](int, int) {});
    if (lane == 0) of_row[row] = n;
  }
  __syncthreads();
  int n = 0;
  for (int r0 = 0; r0 < a.rows; r0 += kThreads) {   // counts to places in the list
    const int r = r0 + threadIdx.x;
    const int mine = r < a.rows ? of_row[r] : 0;
    int total;
    const int before = n + block_sum(mine, s, &total);
    if (r < a.rows) of_row[r] = mine ? before : -1;
    n += total;
  }
  __syncthreads();
  for (int row = wave; row < a.rows; row += kWaves) {
    const int at = of_row[row];
    if (at >= 0) lacking(row, [&](int i, int j) { miss[at + j] = row * a.max_pages + i; });
  }
  __syncthreads();
  const int got = take_free(a, n, s, [&](int j, int p) {
    a.refs[p] = 1;
    a.table[miss[j]] = p;
  });
  if (threadIdx.x == 0) {
    a.info[0] = got;
    a.info[1] = n - got;
  }
}

// scratch: [0] copies, [4..] src pages, dst pages and pairs of the incomplete
// pages (n each), then per row: is a src; the first pair that names it as dst.
__global__ __launch_bounds__(kThreads) void k_pages_fork(PagesArgs a) {
  __shared__ int s[kSlices * kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int* count = a.scratch;
  int* from = count + 4;
  int* to = from + a.n;
  int* pair = to + a.n;
  int* is_src = pair + a.n;
  int* first = is_src + a.rows;
  for (int r = threadIdx.x; r < a.rows; r += kThreads) {
    is_src[r] = 0;
    first[r] = a.n;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < a.n; j += kThreads) {
    const int x = a.src[j], y = a.dst[j];
    if (x >= 0 && x < a.rows) is_src[x] = 1;
    if (y >= 0 && y < a.rows) atomicMin(&first[y], j);
  }
  __syncthreads();
  auto valid = [&](int j) {
    const int x = a.src[j], y = a.dst[j];
    return x >= 0 && x < a.rows && y >= 0 && y < a.rows && fresh(&first[y]) == j && !is_src[y];
  };
  // Complete pages are shared; a wave takes a pair.
  for (int j = wave; j < a.n; j += kWaves) {
    if (!valid(j)) continue;
    const int x = a.src[j], full = held(a, x) >> a.page_log2;
    const int32_t* f = a.table + (int64_t)x * a.max_pages;
    int32_t* t = a.table + (int64_t)a.dst[j] * a.max_pages;
    for (int i0 = 0; i0 < a.max_pages; i0 += 256) {
      int p[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 64 + lane;
        p[u] = i < full ? f[i] : -1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 64 + lane;
        if (i >= a.max_pages) continue;
        if (is_page(a, p[u])) atomicAdd(&a.refs[p[u]], 1);
        else p[u] = -1;
        t[i] = p[u];
      }
    }
  }
  // Pairs with an incomplete last page.
  int n = 0, forked = 0;
  for (int j0 = 0; j0 < a.n; j0 += kThreads) {
    const int j = j0 + threadIdx.x;
    const bool ok = j < a.n && valid(j);
    bool part = false;
    if (ok) {
      const int len = held(a, a.src[j]);
      part = (len & ((1 << a.page_log2) - 1)) &&
             is_page(a, a.table[(int64_t)a.src[j] * a.max_pages + (len >> a.page_log2)]);
      a.lens[a.dst[j]] = len;
    }
    int total;   // both counts in one sum
    const int rank = n + (block_sum(part | ok << 16, s, &total) & 0xffff);
    if (part) pair[rank] = j;
    n += total & 0xffff;
    forked += total >> 16;
  }
  __syncthreads();
  const int got = take_free(a, n, s, [&](int r, int p) {
    const int j = pair[r], x = a.src[j], full = held(a, x) >> a.page_log2;
    from[r] = a.table[(int64_t)x * a.max_pages + full];
    to[r] = p;
    a.refs[p] = 1;
    a.table[(int64_t)a.dst[j] * a.max_pages + full] = p;
  });
  for (int r = got + threadIdx.x; r < n; r += kThreads) {
    const int y = a.dst[pair[r]];
    a.lens[y] = a.lens[y] >> a.page_log2 << a.page_log2;
  }
  if (threadIdx.x == 0) {
    *count = got;
    a.info[0] = forked;
    a.info[1] = n - got;
  }
}

// scratch: per row the first place that names it.  A wave takes a row.
__global__ __launch_bounds__(kThreads) void k_pages_release(PagesArgs a) {
  __shared__ int s_info[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int* first = a.scratch;
  if (threadIdx.x < 2) s_info[threadIdx.x] = 0;
  for (int r = threadIdx.x; r < a.rows; r += kThreads) first[r] = a.n;
  __syncthreads();
  for (int j = threadIdx.x; j < a.n; j += kThreads) {
    const int x = a.src[j];
    if (x >= 0 && x < a.rows) atomicMin(&first[x], j);
  }
  __syncthreads();
  int dropped = 0, freed = 0;
  for (int j = wave; j < a.n; j += kWaves) {
    const int x = a.src[j];
    if (x < 0 || x >= a.rows || fresh(&first[x]) != j) continue;
    int32_t* t = a.table + (int64_t)x * a.max_pages;
    for (int i0 = 0; i0 < a.max_pages; i0 += 256) {
      int p[4], was[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 64 + lane;
        p[u] = i < a.max_pages ? t[i] : -1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) was[u] = is_page(a, p[u]) ? atomicSub(&a.refs[p[u]], 1) : 2;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * 64 + lane;
        if (i < a.max_pages) t[i] = -1;
        if (!is_page(a, p[u])) continue;
        if (was[u] <= 0) atomicAdd(&a.refs[p[u]], 1);   // named by more entries than it had references
        dropped += 1;
        freed += was[u] == 1;
      }
    }
    if (lane == 0) a.lens[x] = 0;
  }
  if (dropped) atomicAdd(&s_info[0], dropped);
  if (freed) atomicAdd(&s_info[1], freed);
  __syncthreads();
  if (threadIdx.x < 2) a.info[threadIdx.x] = s_info[threadIdx.x];
}

// scratch: [0] copies, [4..] src pages, dst pages, then where each page goes.
__global__ __launch_bounds__(kThreads) void k_pages_compact(PagesArgs a) {
  __shared__ int s[kSlices * kWaves];
  int* count = a.scratch;
  int* from = count + 4;
  int* to = from + a.pages;
  int* map = to + a.pages;
  int live = 0;
  for (int p = threadIdx.x; p < a.pages; p += kThreads) {
    const int r = a.refs[p];
    map[p] = p;
    a.refs_out[p] = r;
    live += r > 0;
  }
  block_sum(live, s, &live);
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < a.pages; p0 += kThreads * kSlices) {
    const int slices = min((a.pages - p0 + kThreads - 1) / kThreads, kSlices);
    bool hole[kSlices], mover[kSlices];
    int rank[kSlices], total;
#pragma unroll
    for (int i = 0; i < kSlices; ++i) {
      const int p = p0 + i * kThreads + threadIdx.x;
      const bool used = p < a.pages && a.refs[p] > 0;
      hole[i] = p < live && !used;
      mover[i] = used && p >= live;
    }
    slice_ranks(hole, slices, s, rank, &total);
#pragma unroll
    for (int i = 0; i < kSlices; ++i)
      if (hole[i]) to[holes + rank[i]] = p0 + i * kThreads + threadIdx.x;
    holes += total;
    slice_ranks(mover, slices, s, rank, &total);
#pragma unroll
    for (int i = 0; i < kSlices; ++i)
      if (mover[i]) from[movers + rank[i]] = p0 + i * kThreads + threadIdx.x;
    movers += total;
  }
  __syncthreads();
  for (int r = threadIdx.x; r < movers; r += kThreads) {
    const int x = from[r], y = to[r];
    map[x] = y;
    a.refs_out[y] = a.refs[x];
  }
  __syncthreads();
  for (int r = threadIdx.x; r < movers; r += kThreads) a.refs_out[from[r]] = 0;
  if (threadIdx.x == 0) {
    *count = movers;
    a.info[0] = live;
    a.info[1] = movers;
  }
}

// Bytes from `f` to `t` by the workgroup, 16 a thread at a time; four loads go
// out before the first store.
__device__ __forceinline__ void copy_bytes(const char* f, char* t, int64_t n) {
  for (int64_t b = threadIdx.x * 16; b < n; b += 4 * 256 * 16) {
    u32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (b + i * 4096 < n) w[i] = *reinterpret_cast<const u32x4*>(f + b + i * 4096);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (b + i * 4096 < n) *reinterpret_cast<u32x4*>(t + b + i * 4096) = w[i];
  }
}

// Workgroup (x, y): pairs x, x + gridDim.x, ... of layer y.  A compaction's
// page table is rewritten by the workgroups of one more y.
__global__ __launch_bounds__(256) void k_pages_copy(CopyArgs a) {
  if ((int)blockIdx.y == a.layers) {
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < a.entries; e += (int64_t)gridDim.x * 256) {
      const int p = a.table[e];
      a.table_out[e] = p >= 0 && p < a.from_pages ? a.map[p] : p;
    }
    return;
  }
  const int n = a.count ? *a.count : a.n;
  for (int j = blockIdx.x; j < n; j += gridDim.x) {
    const int x = a.src[j], y = a.dst[j];
    if (x < 0 || x >= a.from_pages || y < 0 || y >= a.to_pages) continue;
    const char* f[4];
    char* t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a.from[i] + blockIdx.y * a.from_layer[i] + x * a.bytes[i];
      t[i] = a.to[i] + blockIdx.y * a.to_layer[i] + y * a.bytes[i];
    }
    copy_bytes(f[0], t[0], a.bytes[0]);
    copy_bytes(f[1], t[1], a.bytes[1]);
    copy_bytes(f[3], t[3], a.bytes[3]);
    for (int64_t b = threadIdx.x * 8; b < a.bytes[2]; b += 256 * 8)   // the scales: 8 bytes a head
      *reinterpret_cast<uint64_t*>(t[2] + b) = *reinterpret_cast<const uint64_t*>(f[2] + b);
  }
}

}  // namespace

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t s) {
  k_pages_reserve<<<1, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t s) {
  k_pages_fork<<<1, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_release(const PagesArgs& a, hipStream_t s) {
  k_pages_release<<<1, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t s) {
  k_pages_compact<<<1, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyArgs& a, hipStream_t s) {
  k_pages_copy<<<dim3(min(a.n, 1024), a.layers + (a.map ? 1 : 0)), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ssba
