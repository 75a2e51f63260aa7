// Drives the cache's host layer (ssba_cache_api.cpp) built for the CPU with
// sanitizers: recording stand-ins for the launchers check what every launch
// would be given, over descriptors at the edges of the integer ranges.
#include <algorithm>
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

namespace {

size_t scratch_given;
char* const kScratch = reinterpret_cast<char*>(0x100000);
int launches;

void check_view(const ssba::CacheView& c, const ssba::BatchView& b) {
  CHECK(c.pages >= 1 && c.kv_heads >= 1 && (c.page_log2 >= 4 && c.page_log2 <= 6));
  CHECK(c.page_bytes == (int64_t)c.kv_heads * c.head_dim << c.page_log2);
  CHECK(b.seqs >= 1 && b.rows >= 1 && b.max_new >= 1 && ((int64_t)b.max_pages << c.page_log2) <= (1 << 30));
}

void check_grid(int64_t groups, int64_t threads) {
  CHECK(groups >= 1 && groups < (int64_t)1 << 31 && groups * threads < (int64_t)1 << 32);
}

}  // namespace

namespace ssba {

hipError_t launch_cache_append(const AppendArgs& a, int, hipStream_t) {
  ++launches;
  check_view(a.c, a.b);
  CHECK(a.slots >= 1);
  check_grid((int64_t)a.b.seqs * a.slots * a.c.kv_heads, 256);
  return hipSuccess;
}

hipError_t launch_cache_select(const SelectArgs& a, const SelectPlan& p, int, hipStream_t) {
  ++launches;
  check_view(a.c, a.b);
  CHECK(a.group >= 1 && a.first >= 0 && a.last >= 1 && a.first + a.last <= a.keep && a.tiles >= 1);
  const int64_t rows = (int64_t)a.b.rows * a.c.kv_heads, tiles = (int64_t)a.b.seqs * a.c.kv_heads * a.tiles;
  CHECK(p.chunks >= 1 && p.chunks <= 65535);
  if (p.kind == kSelectRow) check_grid(rows, 512);
  if (p.kind == kSelectTile) check_grid(tiles, 512);
  if (p.kind <= kSelectTile) CHECK(a.b.max_pages <= kSelectInLds);
  if (p.kind == kSelectRowLong) check_grid(rows * p.chunks, 256);
  if (p.kind == kSelectTileLong) check_grid(tiles * p.chunks, 512);
  if (p.kind >= kSelectRowLong) {
    check_grid(rows, 1024);
    if (p.scored) CHECK((size_t)rows * a.b.max_pages * 8 <= scratch_given && (char*)a.keys == kScratch);
  }
  return hipSuccess;
}

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int, hipStream_t) {
  ++launches;
  check_view(a.c, a.b);
  CHECK(a.group >= 1 && a.splits == p.splits && a.col_tiles == p.col_tiles && p.splits >= 1 && p.splits <= 256);
  check_grid(p.items * p.splits, p.threads);
  check_grid(p.items * p.tiles * (a.c.head_dim / 32), p.splits > 1 ? 256 : 1);
  const int64_t cols = a.lists ? a.group : (int64_t)a.group * a.b.max_new;
  CHECK((int64_t)p.col_tiles * p.tiles * 16 >= cols && cols <= (int64_t)1 << 30);
  if (p.kind == kAttendRows) CHECK(p.splits == 1);
  if (p.splits > 1) {
    const size_t columns = (size_t)p.items * p.splits * p.tiles * 16;
    CHECK((char*)a.part == kScratch && a.part_ml == a.part + columns * a.c.head_dim);
    CHECK((char*)(a.part_ml + columns * 2) <= kScratch + scratch_given);
  }
  return hipSuccess;
}

void check_pages(const PagesArgs& a) {
  ++launches;
  CHECK(a.rows >= 1 && a.pages >= 1 && a.n >= 0 && (int64_t)a.rows * a.max_pages < (int64_t)1 << 31);
  CHECK((char*)a.scratch == kScratch);
}

hipError_t launch_pages_reserve(const PagesArgs& a, hipStream_t) {
  check_pages(a);
  CHECK(4 * ((size_t)a.rows * a.max_pages + a.rows) <= scratch_given);
  return hipSuccess;
}
hipError_t launch_pages_fork(const PagesArgs& a, hipStream_t) {
  check_pages(a);
  CHECK(4 * (4 + (size_t)3 * a.n + (size_t)2 * a.rows) <= scratch_given);
  return hipSuccess;
}
hipError_t launch_pages_release(const PagesArgs& a, hipStream_t) {
  check_pages(a);
  CHECK(4 * (size_t)a.rows <= scratch_given);
  return hipSuccess;
}
hipError_t launch_pages_compact(const PagesArgs& a, hipStream_t) {
  check_pages(a);
  CHECK(4 * (4 + (size_t)3 * a.pages) <= scratch_given);
  return hipSuccess;
}
hipError_t launch_pages_copy(const CopyArgs& a, hipStream_t) {
  ++launches;
  CHECK(a.n >= 1 && a.layers >= 1 && a.layers < 65535 && a.src && a.dst);
  for (int i = 0; i < 4; ++i) CHECK(a.bytes[i] % (i == 2 ? 8 : 16) == 0 && a.from_layer[i] == a.bytes[i] * a.from_pages);
  return hipSuccess;
}

}  // namespace ssba

int main() {
  std::mt19937 rng(1);
  auto pick = [&](std::initializer_list<int> v) { return *(v.begin() + rng() % v.size()); };
  auto p = [&](size_t align) { return rng() % 40 ? reinterpret_cast<void*>((size_t)0x1000 * align) : nullptr; };
  int ok = 0;
  for (int it = 0; it < 60000; ++it) {
    ssba_cache c;
    std::memset(&c, 0, sizeof(c));
    c.layers = pick({1, 2, 24, 65534, 65535, 0, -1});
    c.pages = pick({1, 7, 1000, 70000, 1 << 24, (1 << 24) + 1, 0});
    c.kv_heads = pick({1, 2, 8, 1024, 1025, 0});
    c.head_dim = pick({64, 128, 64, 128, 96, 0});
    c.page = pick({16, 32, 64, 64, 8, 128});
    c.k = p(16);
    c.v = p(16);
    c.scale = (float*)p(16);
    c.kmean = p(16);
    ssba_cache_batch b;
    std::memset(&b, 0, sizeof(b));
    b.seqs = pick({1, 2, 64, 1000, 65535, 65536, 0});
    b.max_pages = pick({1, 5, 1000, 1024, 1025, 5000, 1 << 20, 1 << 24, 1 << 26, 2147483647, 0});
    b.rows = pick({0, 1, 64, 5000, 1 << 20, 1 << 30, 2147483647, -1});
    b.max_new = pick({0, 1, 7, 8, 300, 100000, 1 << 30, 2147483647, -1});
    b.max_len = pick({0, 1, 4000, 1 << 20, 2147483647, -1});
    b.table = (int32_t*)p(4);
    b.lens = (int32_t*)p(4);
    b.cu = (int32_t*)p(4);
    ssba_cache_query q;
    std::memset(&q, 0, sizeof(q));
    q.heads = (int)std::min<int64_t>((int64_t)c.kv_heads * pick({1, 2, 4, 17, 65536}), 2147483647);
    q.dtype = pick({0, 1, 0, 1, 2});
    q.causal = pick({0, 1, 1, 2});
    q.keep = pick({0, 1, 3, 32, 1000, 1 << 24, 2147483647, -1});
    q.first = pick({0, 1, 2, 2147483647, -1});
    q.last = pick({1, 1, 2, 2147483647, 0});
    size_t need = 0;
    const int layer = pick({0, 0, 1, -1, 70000});
    const size_t lists = SIZE_MAX;
    ok += ssba_cache_append(&c, layer, &b, q.dtype, p(16), p(16), 0, 0, nullptr) == SSBA_OK;
    if (ssba_cache_select_workspace_size(&c, &b, &q, &need) == SSBA_OK) {
      scratch_given = need;
      ok += ssba_cache_select(&c, layer, &b, &q, p(16), (int32_t*)p(4), lists, kScratch, need, nullptr) == SSBA_OK;
      if (need) CHECK(ssba_cache_select(&c, layer, &b, &q, p(16), (int32_t*)p(4), lists, kScratch, need - 1, nullptr) != SSBA_OK || b.rows == 0 || b.max_new == 0);
    }
    for (int with = 0; with < 2; ++with) {
      if (ssba_cache_attend_workspace_size(&c, &b, &q, with, &need) != SSBA_OK) continue;
      scratch_given = need;
      const int32_t* l = with ? (const int32_t*)0x4000 : nullptr;
      ok += ssba_cache_attend(&c, layer, &b, &q, p(16), l, lists, p(16), kScratch, need, nullptr) == SSBA_OK;
      if (need) CHECK(ssba_cache_attend(&c, layer, &b, &q, p(16), l, lists, p(16), kScratch, need - 1, nullptr) != SSBA_OK || b.rows == 0 || b.max_new == 0);
    }
    ssba_pages t;
    std::memset(&t, 0, sizeof(t));
    t.rows = pick({1, 3, 1000, 1 << 16, 2147483647, 0});
    t.max_pages = pick({1, 9, 4000, 1 << 15, 1 << 26, 2147483647, 0});
    t.table = (int32_t*)p(4);
    t.lens = (int32_t*)p(4);
    t.refs = (int32_t*)p(4);
    const int n = pick({0, 1, 5, 1000, 1 << 24, 2147483647, -1});
    int32_t* x = (int32_t*)p(4);
    if (ssba_pages_workspace_size(&c, &t, std::max(n, 0), &need) == SSBA_OK) {
      scratch_given = need;
      ok += ssba_pages_reserve(&c, &t, x, kScratch, need, nullptr) == SSBA_OK;
      ok += ssba_pages_fork(&c, &t, n, x, x, x, kScratch, need, nullptr) == SSBA_OK;
      ok += ssba_pages_release(&c, &t, n, x, x, kScratch, need, nullptr) == SSBA_OK;
      ok += ssba_pages_compact(&c, &t, x, x, x, kScratch, need, nullptr) == SSBA_OK;
      CHECK(ssba_pages_reserve(&c, &t, x, kScratch, 3, nullptr) != SSBA_OK);
    }
    ok += ssba_pages_copy(&c, &c, n, x, x, nullptr) == SSBA_OK;
  }
  CHECK(ok > 5000 && launches > 5000);
  std::puts("ok");
  return 0;
}
