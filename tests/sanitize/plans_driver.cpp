// Drives the host layers of the windowed attention's backward and of the shared
// prefixes, built for the CPU with sanitizers: recording stand-ins for the
// launchers check what a launch's workgroups would read and write of the scratch,
// part by part, where several of them share a tile's heads and queries and where
// the prefixes' column tiles are packed.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <set>
#include <vector>

#include "ssba_cache_common.h"
#include "ssba_common.h"
#include "ssba_rope_common.h"
#include "ssba_window_common.h"

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("failed: %s (line %d)\n", #x, __LINE__);             \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

namespace {

size_t scratch_given;
char* const kScratch = reinterpret_cast<char*>(0x100000);
int by_heads, by_queries, by_both, cut_and_shared, whole, packed, unpacked, in_parts;
std::mt19937 rng(3);

void check_grid(int64_t groups, int64_t threads) {
  CHECK(groups >= 0 && groups < (int64_t)1 << 31 && groups * threads < (int64_t)1 << 32);
}

bool inside(const void* p, int64_t bytes) {
  const char* c = static_cast<const char*>(p);
  return c >= kScratch && bytes >= 0 && c + bytes <= kScratch + scratch_given;
}

}  // namespace

namespace ssba {

hipError_t launch_window_forward(const WindowArgs&, int, int, hipStream_t) { return hipSuccess; }

hipError_t launch_window_backward(const WindowArgs& a, int d, int, hipStream_t) {
  CHECK(a.head_parts >= 1 && a.query_parts >= 1 && a.group % a.head_parts == 0);
  const int64_t units = (int64_t)a.batch * a.kv_heads, cut = (int64_t)a.sink_tiles * a.chunk_slots;
  const int64_t shares = (int64_t)a.head_parts * a.query_parts, kept = cut + (shares > 1 ? a.slots : 0);
  check_grid(units * (a.slots + cut) * shares, 256);
  check_grid(units * kept * (kWindowRows * d / 2048), 256);
  const int64_t rows = (int64_t)a.batch * a.heads * a.seq;
  CHECK(inside(a.lse2, rows * 4) && inside(a.ndelta, rows * 4) && a.ndelta >= a.lse2 + rows && a.part >= a.ndelta + rows);
  // The part of the last share of the last tile or chunk that leaves one, and the join's reads of its tile: dk, then dv.
  const int64_t part = 2 * kWindowRows * d;
  if (kept) CHECK(inside(a.part + (((units - 1) * kept + kept - 1) * shares + shares - 1) * part, part * 4));
  // A cut tile's parts begin with its first chunk's; those of a sequence that begins at row b are its chunk slots from
  // b / chunk + s on, as many as it has chunks.
  if (a.chunk_slots) {
    for (int it = 0; it < 4; ++it) {
      const int seqs = std::max(a.seqs, 1), s = rng() % seqs;
      const int64_t begin = a.seqs ? rng() % (uint64_t)(a.seq + 1) : 0, len = a.seqs ? rng() % (uint64_t)(a.seq - begin + 1) : a.seq;
      if (!len) continue;
      const int64_t first = a.seqs ? begin / a.chunk + s : 0, chunks = (len + a.chunk - 1) / a.chunk;
      CHECK(first + chunks <= a.chunk_slots);
    }
  }
  by_heads += a.head_parts > 1;
  by_queries += a.query_parts > 1;
  by_both += a.head_parts > 1 && a.query_parts > 1;
  cut_and_shared += a.chunk_slots && shares > 1;
  whole += !kept;
  return hipSuccess;
}

hipError_t launch_rope_turn(const TurnArgs&, int, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_append(const AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_select(const SelectArgs&, const SelectPlan&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_reserve(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_fork(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_release(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_compact(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_copy(const CopyArgs&, hipStream_t) { return hipSuccess; }

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int, hipStream_t) {
  CHECK(p.kind == kAttendShared && a.prefix_slots == p.prefix_slots && p.prefix_splits >= 1);
  const int64_t d = a.c.head_dim, w = a.prefix_cols, kv = a.c.kv_heads;
  CHECK(w >= 16 && w <= 256 && (w & (w - 1)) == 0);      // kernels shift by its logarithm
  check_grid(p.prefix_items * p.prefix_splits, p.prefix_threads);
  check_grid(p.items * p.splits, p.threads);
  // Column col of part s of item i: its sums and its maximum.
  auto slot = [&](int64_t item, int64_t s, int64_t col) { return (item * p.prefix_splits + s) * w + col; };
  auto there = [&](int64_t x) { return inside(a.prefix_part + x * d, d * 4) && inside(a.prefix_ml + x * 2, 8); };
  in_parts += p.splits > 1;
  if (!a.prefix_slots) {
    ++unpacked;
    CHECK(p.prefix_items == (int64_t)a.groups * kv * a.prefix_col_tiles && (int64_t)a.prefix_col_tiles * w >= a.shared_cols);
    CHECK(there(slot(p.prefix_items - 1, p.prefix_splits - 1, w - 1)));
    return hipSuccess;
  }
  ++packed;
  CHECK(p.prefix_items == (int64_t)a.prefix_slots * kv);
  CHECK(there(slot(p.prefix_items - 1, p.prefix_splits - 1, w - 1)));
  // Groups of rows that do not decrease: their tiles are there, and no two have one in common.
  const int groups = std::min(a.groups, 2000);
  std::vector<int64_t> first(groups + 1);
  for (auto& x : first) x = rng() % ((uint64_t)a.b.rows + 1);
  std::sort(first.begin(), first.end());
  if (rng() % 4 == 0) std::fill(first.begin(), first.end() - 1, 0), first.back() = a.b.rows;
  int64_t next = 0;
  for (int g = 0; g < groups; ++g) {
    const int64_t at = first[g] * a.group / w + g, cols = (first[g + 1] - first[g]) * a.group;
    CHECK(at >= next);
    next = at + (cols + w - 1) / w;
    CHECK(next <= a.prefix_slots);
  }
  return hipSuccess;
}

}  // namespace ssba

int main() {
  auto pick = [&](std::initializer_list<int> v) { return *(v.begin() + rng() % v.size()); };
  auto some = [&](double most) { return (int)std::lround(std::exp(std::log(most) * (rng() / 4294967296.0))); };
  for (int it = 0; it < 60000; ++it) {
    ssba_window w;
    std::memset(&w, 0, sizeof(w));
    const bool is_packed = rng() % 2;
    w.batch = is_packed ? 1 : some(8);
    w.seq = some(rng() % 8 ? 20000 : 1 << 24);
    w.kv_heads = some(16);
    w.heads = w.kv_heads * pick({1, 2, 3, 4, 6, 8, 16});
    w.head_dim = pick({64, 128});
    w.dtype = pick({0, 1});
    w.window = some(10000);
    w.sinks = pick({0, 0, 1, 4, 130, 1000});
    w.seqs = is_packed ? some(300) : 0;
    w.max_len = pick({0, 0, 1, 300, 5000, 2147483647});
    w.cu = is_packed ? reinterpret_cast<const int32_t*>(0x4000) : nullptr;
    ssba_window_grads g;
    std::memset(&g, 0, sizeof(g));
    void* x = reinterpret_cast<void*>(0x10000);
    size_t need = 0;
    if (ssba_window_backward_workspace_size(&w, &need) == SSBA_OK) {
      auto call = [&](size_t bytes) {
        scratch_given = bytes;
        return ssba_window_backward(&w, &g, x, x, x, x, x, static_cast<float*>(x), x, x, x, kScratch, bytes, nullptr);
      };
      CHECK(call(need) == SSBA_OK);
      CHECK(call(need - 1) == SSBA_ERR_WORKSPACE);
    }

    ssba_cache c;
    std::memset(&c, 0, sizeof(c));
    c.layers = 1;
    c.pages = 1 << 20;
    c.kv_heads = some(16);
    c.head_dim = pick({64, 128});
    c.page = pick({16, 32, 64});
    c.k = c.v = c.kmean = x;
    c.scale = static_cast<float*>(x);
    ssba_cache_batch b;
    std::memset(&b, 0, sizeof(b));
    b.seqs = some(rng() % 8 ? 300 : 65535);
    b.max_pages = some(1 << 14);
    b.max_new = some(rng() % 4 ? 16 : 4000);
    b.rows = (int)std::min<int64_t>((int64_t)b.seqs * b.max_new, 1 << 24) / pick({1, 1, 2, 7}) + pick({0, 0, 5});
    b.max_len = pick({0, 1, 3000, 200000});
    b.table = b.lens = b.cu = static_cast<int32_t*>(x);
    ssba_cache_query q;
    std::memset(&q, 0, sizeof(q));
    q.heads = c.kv_heads * pick({1, 2, 4, 7, 16});
    q.dtype = pick({0, 1});
    q.causal = pick({0, 1});
    const int groups = std::min(some(65535), b.seqs);
    ssba_cache_prefix pre = {groups, rng() % 2 ? b.seqs : std::max(1, b.seqs / groups), pick({0, 0, 1, 4096, 1 << 20}),
                             static_cast<int32_t*>(x), static_cast<int32_t*>(x)};
    if (ssba_cache_attend_shared_workspace_size(&c, &b, &q, &pre, &need) == SSBA_OK && b.rows) {
      auto call = [&](size_t bytes) {
        scratch_given = bytes;
        return ssba_cache_attend_shared(&c, 0, &b, &q, &pre, x, x, kScratch, bytes, nullptr);
      };
      CHECK(call(need) == SSBA_OK);
      CHECK(call(need - 1) == SSBA_ERR_WORKSPACE);
    }
  }
  std::fprintf(stderr, "heads %d queries %d both %d cut %d whole %d packed %d unpacked %d parts %d\n", by_heads, by_queries,
               by_both, cut_and_shared, whole, packed, unpacked, in_parts);
  CHECK(by_heads > 1000 && by_queries > 1000 && by_both > 300 && cut_and_shared > 300 && whole > 1000);
  CHECK(packed > 1000 && unpacked > 1000 && in_parts > 1000);
  std::puts("ok");
  return 0;
}
