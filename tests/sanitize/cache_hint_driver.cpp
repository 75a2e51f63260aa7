// Drives the cache's host layer (ssba_cache_api.cpp) built for the CPU: whether
// a call is accepted must not depend on max_len, by which only work is split.
// Stand-ins for the launchers check the grids of what is accepted.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "ssba_cache_common.h"
#include "ssba_common.h"

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("failed: %s (line %d)\n", #x, __LINE__);             \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)

namespace ssba {

static void grid(int64_t groups, int64_t threads) {
  CHECK(groups >= 1 && groups < (int64_t)1 << 31 && groups * threads < (int64_t)1 << 32);
}

hipError_t launch_cache_append(const AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_select(const SelectArgs& a, const SelectPlan& p, int, hipStream_t) {
  const int64_t rows = (int64_t)a.b.rows * a.c.kv_heads, tiles = (int64_t)a.b.seqs * a.c.kv_heads * a.tiles;
  const bool tile = p.kind == kSelectTile || p.kind == kSelectTileLong;
  CHECK(p.chunks >= 1 && p.chunks <= 65535);
  grid((tile ? tiles : rows) * p.chunks, tile || p.kind == kSelectRow ? 512 : 256);
  if (p.kind >= kSelectRowLong) grid(rows, 1024);
  return hipSuccess;
}
hipError_t launch_cache_attend(const AttendArgs&, const AttendPlan& p, int, hipStream_t) {
  grid(p.items * p.splits, p.threads);
  return hipSuccess;
}
hipError_t launch_pages_reserve(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_fork(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_release(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_compact(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_copy(const CopyArgs&, hipStream_t) { return hipSuccess; }

}  // namespace ssba

int main() {
  std::mt19937 rng(2);
  auto pick = [&](std::initializer_list<int> v) { return *(v.begin() + rng() % v.size()); };
  auto at = [](size_t x) { return reinterpret_cast<void*>(x); };
  int accepted = 0, refused = 0;
  auto same = [&](int kv, int rows, int seqs, int max_new, int max_pages, int keep) {
    ssba_cache c;
    std::memset(&c, 0, sizeof(c));
    c.layers = 1;
    c.pages = 70000;
    c.kv_heads = kv;
    c.head_dim = 64;
    c.page = 16;
    c.k = c.v = c.kmean = at(0x1000);
    c.scale = static_cast<float*>(at(0x1000));
    ssba_cache_batch b;
    std::memset(&b, 0, sizeof(b));
    b.seqs = seqs;
    b.max_pages = max_pages;
    b.rows = rows;
    b.max_new = max_new;
    b.table = b.lens = b.cu = static_cast<int32_t*>(at(0x1000));
    ssba_cache_query q;
    std::memset(&q, 0, sizeof(q));
    q.heads = c.kv_heads;
    q.causal = 1;
    q.keep = keep;
    q.first = q.last = 1;
    int first[3] = {0, 0, 0};
    for (int hint : {4096, 0, 1, 1 << 20, 2147483647}) {
      b.max_len = hint;
      const int32_t* lists = rng() % 2 ? static_cast<int32_t*>(at(0x4000)) : nullptr;
      const int got[3] = {
          ssba_cache_append(&c, 0, &b, 0, at(0x1000), at(0x1000), 0, 0, nullptr),
          ssba_cache_select(&c, 0, &b, &q, at(0x1000), static_cast<int32_t*>(at(0x4000)), SIZE_MAX, at(0x1000), SIZE_MAX,
                            nullptr),
          lists ? 0 : ssba_cache_attend(&c, 0, &b, &q, at(0x1000), nullptr, 0, at(0x8000), at(0x1000), SIZE_MAX, nullptr)};
      for (int i = 0; i < 3; ++i) {
        if (hint == 4096) first[i] = i == 2 && lists ? -1 : got[i];
        if (i == 2 && (lists || first[i] < 0)) continue;
        if (got[i] != first[i])
          std::printf("call %d, max_len %d: %d, with 4096 %d; kv %d rows %d seqs %d new %d pages %d\n", i, hint, got[i],
                      first[i], c.kv_heads, b.rows, b.seqs, b.max_new, b.max_pages);
        CHECK(got[i] == first[i]);
        (got[i] == SSBA_OK ? accepted : refused) += 1;
      }
    }
    return first[1];
  };
  // one call whose hint must not matter, single tokens and tiles of them
  CHECK(same(16, 1024, 1024, 1, 65536, 8) == SSBA_OK);
  CHECK(same(16, 4096, 8, 512, 1 << 20, 8) == SSBA_OK);
  for (int it = 0; it < 20000; ++it)
    same(pick({1, 2, 16, 128, 1024}), pick({1, 64, 1024, 5000, 1 << 18, 1 << 22, 1 << 30}), pick({1, 4, 64, 1024, 65535}),
         pick({1, 7, 8, 40, 3000, 1 << 20}), pick({1, 1000, 1153, 4096, 65536, 1 << 22, 1 << 26}), pick({2, 32, 5000}));
  CHECK(accepted > 20000 && refused > 5000);
  std::puts("ok");
  return 0;
}
