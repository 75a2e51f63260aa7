// Page bookkeeping of the cache (include/ssba_cache.h): one workgroup walks
// the small arrays (references, page table) and leaves a list of page copies;
// a second launch moves the pages of all layers.
#include <hip/hip_runtime.h>

#include "ssba_cache.h"

namespace ssba {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;

// Number of set flags in front of this thread's, and their total, over the
// workgroup.  `s` is LDS of kWaves ints.
__device__ __forceinline__ int block_rank(bool flag, int* s, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t m = __builtin_amdgcn_ballot_w64(flag);
  __syncthreads();
  if (lane == 0) s[wave] = __popcll(m);
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? s[w] : 0;
    sum += s[w];
  }
  *total = sum;
  return before + __popcll(m & ((1ull << lane) - 1));
}

__device__ __forceinline__ int held(const PagesArgs& a, int row) {
  return min(max(a.lens[row], 0), a.max_pages << a.page_log2);
}

__device__ __forceinline__ bool is_page(const PagesArgs& a, int p) { return p >= 0 && p < a.pages; }

// Read past the L1, which this kernel's own atomics do not update.
__device__ __forceinline__ int fresh(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The lowest `n` free pages, in order: fn(j, page) for j < n; returns how many there are (at most n).
template <typename F>
__device__ __forceinline__ int take_free(const PagesArgs& a, int n, int* s, F fn) {
  int got = 0;
  for (int p0 = 0; p0 < a.pages && got < n; p0 += kThreads) {
    const int p = p0 + threadIdx.x;
    int total;
    const bool free = p < a.pages && fresh(&a.refs[p]) == 0;
    const int rank = got + block_rank(free, s, &total);
    if (free && rank < n) fn(rank, p);
    got += total;
  }
  return min(got, n);
}

__global__ __launch_bounds__(kThreads) void k_pages_reserve(PagesArgs a) {
  __shared__ int s[kWaves];
  int* miss = a.scratch;
  int n = 0;
  const int64_t entries = (int64_t)a.rows * a.max_pages;
  for (int64_t e0 = 0; e0 < entries; e0 += kThreads) {
    const int64_t e = e0 + threadIdx.x;
    bool lacks = false;
    if (e < entries) {
      const int row = (int)(e / a.max_pages), i = (int)(e - (int64_t)row * a.max_pages);
      lacks = (i << a.page_log2) < held(a, row) && !is_page(a, a.table[e]);
    }
    int total;
    const int rank = n + block_rank(lacks, s, &total);
    if (lacks) miss[rank] = (int)e;
    n += total;
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

// scratch: [0] copies, then src and dst pages of the copies (n each), then
// per row: is a src; the first pair that names it as dst; then per pair the
// rank of its incomplete page.
__global__ __launch_bounds__(kThreads) void k_pages_fork(PagesArgs a) {
  __shared__ int s[kWaves];
  int* count = a.scratch;
  int* from = count + 4;
  int* to = from + a.n;
  int* pair = to + a.n;        // of the j-th incomplete page
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
  // Complete pages are shared.
  const int64_t entries = (int64_t)a.n * a.max_pages;
  for (int64_t e = threadIdx.x; e < entries; e += kThreads) {
    const int j = (int)(e / a.max_pages), i = (int)(e - (int64_t)j * a.max_pages);
    if (!valid(j)) continue;
    const int x = a.src[j];
    int p = -1;
    if (i < held(a, x) >> a.page_log2) {
      p = a.table[(int64_t)x * a.max_pages + i];
      if (is_page(a, p)) atomicAdd(&a.refs[p], 1);
      else p = -1;
    }
    a.table[(int64_t)a.dst[j] * a.max_pages + i] = p;
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
    int total;
    const int rank = n + block_rank(part, s, &total);
    if (part) pair[rank] = j;
    n += total;
    block_rank(ok, s, &total);
    forked += total;
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

// scratch: per row the first place that names it.
__global__ __launch_bounds__(kThreads) void k_pages_release(PagesArgs a) {
  __shared__ int s_info[2];
  int* first = a.scratch;
  if (threadIdx.x < 2) s_info[threadIdx.x] = 0;
  for (int r = threadIdx.x; r < a.rows; r += kThreads) first[r] = a.n;
  __syncthreads();
  for (int j = threadIdx.x; j < a.n; j += kThreads) {
    const int x = a.src[j];
    if (x >= 0 && x < a.rows) atomicMin(&first[x], j);
  }
  __syncthreads();
  const int64_t entries = (int64_t)a.n * a.max_pages;
  int dropped = 0, freed = 0;
  for (int64_t e = threadIdx.x; e < entries; e += kThreads) {
    const int j = (int)(e / a.max_pages), i = (int)(e - (int64_t)j * a.max_pages);
    const int x = a.src[j];
    if (x < 0 || x >= a.rows || fresh(&first[x]) != j) continue;
    int32_t* at = a.table + (int64_t)x * a.max_pages + i;
    const int p = *at;
    if (is_page(a, p)) {
      const int was = atomicSub(&a.refs[p], 1);
      if (was <= 0) atomicAdd(&a.refs[p], 1);   // named by more entries than it had references
      dropped += 1;
      freed += was == 1;
    }
    *at = -1;
    if (i == 0) a.lens[x] = 0;
  }
  if (dropped) atomicAdd(&s_info[0], dropped);
  if (freed) atomicAdd(&s_info[1], freed);
  __syncthreads();
  if (threadIdx.x < 2) a.info[threadIdx.x] = s_info[threadIdx.x];
}

// scratch: [0] copies, [4..] src pages, dst pages, then where each page goes.
__global__ __launch_bounds__(kThreads) void k_pages_compact(PagesArgs a) {
  __shared__ int s[kWaves];
  int* count = a.scratch;
  int* from = count + 4;
  int* to = from + a.pages;
  int* map = to + a.pages;
  int live = 0;
  for (int p0 = 0; p0 < a.pages; p0 += kThreads) {
    const int p = p0 + threadIdx.x;
    const int r = p < a.pages ? a.refs[p] : 0;
    if (p < a.pages) {
      map[p] = p;
      a.refs_out[p] = r;
    }
    int total;
    block_rank(r > 0, s, &total);
    live += total;
  }
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < a.pages; p0 += kThreads) {
    const int p = p0 + threadIdx.x;
    const bool used = p < a.pages && a.refs[p] > 0;
    const bool hole = p < live && !used, mover = used && p >= live;
    int total;
    int rank = holes + block_rank(hole, s, &total);
    holes += total;
    if (hole) to[rank] = p;
    rank = movers + block_rank(mover, s, &total);
    movers += total;
    if (mover) from[rank] = p;
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
