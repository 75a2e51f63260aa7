// Drives the host layers of the windowed attention, the rotary positions and
// the cache's windows and shared prefixes, built for the CPU with sanitizers:
// recording stand-ins for the launchers check what every launch would be given,
// over descriptors at the edges of the integer ranges.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

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
int windows, backwards, ropes, cached, shared;

void check_grid(int64_t groups, int64_t threads) {
  CHECK(groups >= 0 && groups < (int64_t)1 << 31 && groups * threads < (int64_t)1 << 32);
}

void check_window(const ssba::WindowArgs& a) {
  CHECK(a.batch >= 1 && a.seq >= 1 && a.kv_heads >= 1 && a.group >= 1 && a.group * a.kv_heads == a.heads);
  CHECK(a.window >= 1 && a.sinks >= 0 && a.sinks <= a.seq && a.scale > 0 && std::isfinite(a.scale_log2));
  CHECK(a.cu ? a.batch == 1 && a.seqs >= 1 : a.seqs == 0);
  CHECK((int64_t)a.slots * ssba::kWindowRows >= a.seq);
  CHECK(a.sink_tiles * (int64_t)ssba::kWindowRows >= a.sinks && a.chunk >= 1024 && a.chunk % ssba::kWindowRows == 0);
  check_grid((int64_t)a.batch * a.heads * a.slots, 256);
  for (const ssba::Strides& s : {a.sq, a.sk, a.sv, a.so})
    CHECK(s.b >= 0 && s.h >= 0 && s.t >= 0 && s.t <= 1 << 20);
}

}  // namespace

namespace ssba {

hipError_t launch_window_forward(const WindowArgs& a, int, int, hipStream_t) {
  ++windows;
  check_window(a);
  return hipSuccess;
}

hipError_t launch_window_backward(const WindowArgs& a, int d, int, hipStream_t) {
  ++backwards;
  check_window(a);
  const int64_t units = (int64_t)a.batch * a.kv_heads, cut = (int64_t)a.sink_tiles * a.chunk_slots;
  const int64_t kept = cut + (a.head_parts > 1 ? a.slots : 0);
  CHECK(a.head_parts >= 1 && a.group % a.head_parts == 0);
  check_grid(units * (a.slots + cut) * a.head_parts, 256);
  check_grid(units * kept * (kWindowRows * d / 2048), 256);
  const int64_t rows = (int64_t)a.batch * a.heads * a.seq;
  CHECK((char*)a.lse2 == kScratch && a.ndelta >= a.lse2 + rows && a.part >= a.ndelta + rows);
  CHECK((char*)(a.part + units * kept * a.head_parts * 2 * kWindowRows * d) <= kScratch + scratch_given);
  // A chunk slot for every chunk that a sequence can have.
  if (a.chunk_slots) CHECK((int64_t)a.chunk_slots * a.chunk >= a.seq);
  return hipSuccess;
}

hipError_t launch_rope_turn(const TurnArgs& a, int d, int, int, hipStream_t) {
  ++ropes;
  CHECK(a.tokens >= 1 && a.rows >= 1 && a.heads[0] >= 1 && a.head_parts >= 1 && a.x[0] && a.y[0]);
  CHECK(a.heads[1] == 0 || (a.x[1] && a.y[1]));
  check_grid((a.tokens + kRopeRows - 1) / kRopeRows * a.head_parts, 256);
  for (int j = 0; j < d / 2; ++j) CHECK(a.axis[j] >= -1 && a.axis[j] < 4 && std::fabs(a.freq[j]) < 1 << 20);
  return hipSuccess;
}

hipError_t launch_cache_append(const AppendArgs&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_cache_select(const SelectArgs&, const SelectPlan&, int, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_reserve(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_fork(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_release(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_compact(const PagesArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_pages_copy(const CopyArgs&, hipStream_t) { return hipSuccess; }

hipError_t launch_cache_attend(const AttendArgs& a, const AttendPlan& p, int, hipStream_t) {
  CHECK(a.group >= 1 && a.splits == p.splits && a.col_tiles == p.col_tiles && p.splits >= 1 && p.splits <= 256);
  check_grid(p.items * p.splits, p.threads);
  check_grid(p.items * p.tiles * (a.c.head_dim / 32), p.splits > 1 ? 256 : 1);
  CHECK((int64_t)p.col_tiles * p.tiles * 16 >= (int64_t)a.group * a.b.max_new);
  const int64_t d = a.c.head_dim, rest = p.splits > 1 ? p.items * p.splits * p.tiles * 16 : 0;
  if (p.kind == kAttendWindow) {
    ++cached;
    CHECK(a.window >= 1 && a.window <= 1 << 30 && a.sinks >= 0 && a.sinks <= 1 << 30);
    if (rest) {
      CHECK((char*)a.part == kScratch && a.part_ml == a.part + rest * d);
      CHECK((char*)(a.part_ml + rest * 2) <= kScratch + scratch_given);
    }
    return hipSuccess;
  }
  CHECK(p.kind == kAttendShared);
  ++shared;
  const int64_t pre = p.prefix_items * p.prefix_splits * p.prefix_tiles * 16;
  CHECK(a.groups >= 1 && a.first && a.shared && a.tiles == p.tiles && p.prefix_splits >= 1 && p.prefix_splits <= 256);
  CHECK(a.prefix_cols == p.prefix_tiles * 16 && a.prefix_col_tiles == p.prefix_col_tiles && a.prefix_splits == p.prefix_splits);
  CHECK((int64_t)a.prefix_col_tiles * a.prefix_cols >= a.shared_cols);
  check_grid(p.prefix_items * p.prefix_splits, p.prefix_threads);
  CHECK((char*)a.part == kScratch && a.prefix_part == a.part + rest * d && a.part_ml == a.prefix_part + pre * d &&
        a.prefix_ml == a.part_ml + rest * 2);
  CHECK((char*)(a.prefix_ml + pre * 2) <= kScratch + scratch_given);
  return hipSuccess;
}

}  // namespace ssba

int main() {
  std::mt19937 rng(1);
  auto pick = [&](std::initializer_list<int> v) { return *(v.begin() + rng() % v.size()); };
  auto p = [&](size_t align) { return rng() % 60 ? reinterpret_cast<void*>((size_t)0x1000 * align) : nullptr; };
  auto strides = [&](int heads, int seq, int d) {
    ssba_strides s = {0, 0, 0};
    if (rng() % 3 == 0) s = {(int64_t)std::min((double)seq * heads * d, 0x1p62), d, (int64_t)heads * d};
    if (rng() % 20 == 0) s.t = pick({1, 7, 8, 64, 1 << 20, (1 << 20) + 8, -8});
    if (rng() % 20 == 0) s.b = pick({0, 8, -8, 2147483640});
    return s;
  };
  for (int it = 0; it < 60000; ++it) {
    ssba_window w;
    std::memset(&w, 0, sizeof(w));
    const bool packed = rng() % 2;
    w.batch = packed ? pick({1, 1, 1, 2, 0}) : pick({1, 2, 8, 1000, 1 << 24, (1 << 24) + 1, 0, -1});
    w.seq = pick({1, 2, 127, 129, 5000, 16384, 1 << 20, 1 << 30, 2147483647, 0, -1});
    w.kv_heads = pick({1, 2, 8, 64, 65536, 0});
    w.heads = (int)std::min<int64_t>((int64_t)w.kv_heads * pick({1, 2, 3, 4, 6, 1000}), 2147483647);
    if (rng() % 30 == 0) w.heads += 1;
    w.head_dim = pick({64, 128, 64, 128, 96});
    w.dtype = pick({0, 1, 0, 1, 2});
    w.window = pick({1, 63, 1024, 5000, 1 << 30, 2147483647, 0});
    w.sinks = pick({0, 0, 4, 200, 5000, 2147483647, -1});
    w.seqs = packed ? pick({1, 2, 64, 5000, 65535, 65536, -1}) : 0;
    w.max_len = pick({0, 0, 100, 5000, 2147483647, -1});
    w.softmax_scale = pick({0, 0, 1, -1}) * (rng() % 50 ? 0.1f : INFINITY);
    w.cu = packed ? (const int32_t*)p(4) : nullptr;
    w.q = strides(w.heads, w.seq, w.head_dim);
    w.k = strides(w.kv_heads, w.seq, w.head_dim);
    w.v = strides(w.kv_heads, w.seq, w.head_dim);
    w.o = strides(w.heads, w.seq, w.head_dim);
    ssba_window_forward(&w, p(16), p(16), p(16), p(16), (float*)p(4), nullptr);
    size_t need = 0;
    const ssba_status st = ssba_window_backward_workspace_size(&w, &need);
    if (st == SSBA_OK) {
      ssba_window_grads g;
      g.do_ = strides(w.heads, w.seq, w.head_dim);
      g.dq = strides(w.heads, w.seq, w.head_dim);
      g.dk = strides(w.kv_heads, w.seq, w.head_dim);
      g.dv = strides(w.kv_heads, w.seq, w.head_dim);
      scratch_given = need;
      CHECK(need < (size_t)1 << 36);
      ssba_window_backward(&w, &g, p(16), p(16), p(16), p(16), p(16), (const float*)p(4), p(16), p(16), p(16), kScratch,
                           need, nullptr);
      if (need) CHECK(ssba_window_backward(&w, &g, p(16), p(16), p(16), p(16), p(16), (const float*)p(4), p(16), p(16),
                                           p(16), kScratch, need - 1, nullptr) != SSBA_OK);
    }

    int32_t axis[64];
    double freq[64];
    for (int j = 0; j < 64; ++j) {
      axis[j] = (int)(rng() % 3) - 1;
      freq[j] = std::pow(10.0, -(double)(rng() % 8));
    }
    if (rng() % 20 == 0) axis[rng() % 64] = pick({-2, 3, 100});
    if (rng() % 20 == 0) freq[rng() % 64] = pick({0, 1, 2}) ? 1e7 : NAN;
    ssba_rope r = {pick({64, 128, 64, 128, 64, 128, 96}), pick({0, 1, 0, 1, 0, 1, 2}), pick({2, 4, 2, 4, 2, 4, 0, 5}), axis, freq};
    if (rng() % 40 == 0) r.axis = nullptr;
    ssba_rope_tensor t[2];
    std::memset(t, 0, sizeof(t));
    const int batch = pick({1, 2, 3, 1000, 2147483647, 0, -1}), rows = pick({1, 5, 77, 16384, 2147483647, 0, -1});
    for (int i = 0; i < 2; ++i) {
      t[i].heads = pick({1, 4, 24, 7, 65536, 1, 2, 3, 65537, 0});
      t[i].x = p(16);
      t[i].y = p(16);
      const ssba_strides x = strides(t[i].heads, rows, r.head_dim);
      t[i].x_stride_b = x.b;
      t[i].x_stride_h = x.h;
      t[i].x_stride_t = x.t;
    }
    ssba_rope_rotate(&r, pick({0, 1, 0, 1, 0, 1, 2}), pick({0, 1, 0, 1, 0, 1, 2}), batch, rows, (const int32_t*)p(4),
                     pick({0, 3, 0, 3, 0, 3, -1}), pick({2, 3, 2, 3, 2, 3, -1}), pick({1, 2, 1, 2, 1, 2, 0, 3}), t, nullptr);

    ssba_cache c;
    std::memset(&c, 0, sizeof(c));
    c.layers = 1;
    c.pages = pick({1, 7, 70000, 1 << 24});
    c.kv_heads = pick({1, 2, 8, 1024});
    c.head_dim = pick({64, 128});
    c.page = pick({16, 32, 64});
    c.k = p(16);
    c.v = p(16);
    c.scale = (float*)p(16);
    c.kmean = p(16);
    ssba_cache_batch b;
    std::memset(&b, 0, sizeof(b));
    b.seqs = pick({1, 2, 64, 1000, 65535});
    b.max_pages = pick({1, 5, 1000, 5000, 1 << 20, 1 << 24});
    b.rows = pick({0, 1, 64, 5000, 1 << 20, 1 << 30});
    b.max_new = pick({0, 1, 7, 300, 100000, 1 << 30});
    b.max_len = pick({0, 1, 4000, 1 << 20, 2147483647});
    b.table = (int32_t*)p(4);
    b.lens = (int32_t*)p(4);
    b.cu = (int32_t*)p(4);
    ssba_cache_query q;
    std::memset(&q, 0, sizeof(q));
    q.heads = (int)std::min<int64_t>((int64_t)c.kv_heads * pick({1, 2, 4, 17}), 2147483647);
    q.dtype = pick({0, 1});
    q.causal = pick({0, 1});
    const int window = pick({1, 100, 4096, 2147483647, 0, -5}), sinks = pick({0, 4, 300, 2147483647, -1});
    if (ssba_cache_attend_window_workspace_size(&c, &b, &q, window, sinks, &need) == SSBA_OK) {
      CHECK(window >= 1 && sinks >= 0);
      scratch_given = need;
      ssba_cache_attend_window(&c, 0, &b, &q, window, sinks, p(16), p(16), kScratch, need, nullptr);
      if (need) CHECK(ssba_cache_attend_window(&c, 0, &b, &q, window, sinks, p(16), p(16), kScratch, need - 1, nullptr) !=
                          SSBA_OK || b.rows == 0 || b.max_new == 0);
    }
    ssba_cache_prefix x = {pick({1, 2, 64, 65535, 65536, 0}), pick({1, 8, 1000, 65535, 65536, 0}),
                           pick({0, 1, 8192, 1 << 20, 2147483647, -1}), (const int32_t*)p(4), (const int32_t*)p(4)};
    if (ssba_cache_attend_shared_workspace_size(&c, &b, &q, &x, &need) == SSBA_OK) {
      scratch_given = need;
      CHECK(need > 0 && need < (size_t)1 << 44);
      ssba_cache_attend_shared(&c, 0, &b, &q, &x, p(16), p(16), kScratch, need, nullptr);
      CHECK(ssba_cache_attend_shared(&c, 0, &b, &q, &x, p(16), p(16), kScratch, need - 1, nullptr) != SSBA_OK ||
            b.rows == 0 || b.max_new == 0);
    }
  }
  std::fprintf(stderr, "launches: %d %d %d %d %d\n", windows, backwards, ropes, cached, shared);
  CHECK(windows > 1000 && backwards > 1000 && ropes > 1000 && cached > 1000 && shared > 1000);
  std::puts("ok");
  return 0;
}
