// C ABI of the paged 8-bit cache: argument checks, workspace sizes and launch
// plans.  See include/ssba_cache.h for the contract.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "ssba_cache_common.h"
#include "ssba_common.h"

namespace {

using ssba::AttendArgs;
using ssba::AttendPlan;
using ssba::BatchView;
using ssba::CacheView;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int ilog2(int v) {
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

constexpr int kMaxPages = 1 << 24;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr float kLog2e = 1.4426950408889634f;

ssba_status check_shape(const ssba_cache* c) {
  if (!c) return SSBA_ERR_ARG;
  if (c->layers < 1 || c->pages < 1 || c->kv_heads < 1) return SSBA_ERR_SHAPE;
  if (c->pages > kMaxPages || c->kv_heads > 1024 || c->layers > 65534) return SSBA_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return SSBA_ERR_UNSUPPORTED;
  if (c->page != 16 && c->page != 32 && c->page != 64) return SSBA_ERR_UNSUPPORTED;
  return SSBA_OK;
}

ssba_status check_arrays(const ssba_cache* c) {
  if (!c->k || !c->v || !c->scale || !c->kmean) return SSBA_ERR_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scale, 8) || !aligned(c->kmean, 16)) return SSBA_ERR_ARG;
  return SSBA_OK;
}

ssba_status check_batch(const ssba_cache* c, const ssba_cache_batch* b) {
  if (!b) return SSBA_ERR_ARG;
  if (b->seqs < 1 || b->max_pages < 1 || b->rows < 0 || b->max_new < 0 || b->max_len < 0) return SSBA_ERR_SHAPE;
  if (b->seqs > 65535) return SSBA_ERR_UNSUPPORTED;
  if ((int64_t)b->max_pages * c->page > kMaxTokens || b->rows > kMaxTokens || b->max_new > kMaxTokens)
    return SSBA_ERR_UNSUPPORTED;
  return SSBA_OK;
}

ssba_status check_batch_arrays(const ssba_cache_batch* b) {
  if (!b->table || !b->lens || !b->cu) return SSBA_ERR_ARG;
  if (!aligned(b->table, 4) || !aligned(b->lens, 4) || !aligned(b->cu, 4)) return SSBA_ERR_ARG;
  return SSBA_OK;
}

// Element strides of a packed [rows][heads][D] array; both 0: contiguous.
ssba_status strides_of(int dtype, int heads, int d, int64_t rows, int64_t* st, int64_t* sh) {
  if (dtype != SSBA_DT_BF16 && dtype != SSBA_DT_F32) return SSBA_ERR_ARG;
  if (*st == 0 && *sh == 0) {
    *sh = d;
    *st = (int64_t)heads * d;
  }
  if (*st < 0 || *sh < 0) return SSBA_ERR_SHAPE;
  if ((rows > 1 && *st < d) || (heads > 1 && *sh < d)) return SSBA_ERR_SHAPE;
  if (dtype == SSBA_DT_BF16 && ((*st | *sh) & 7)) return SSBA_ERR_UNSUPPORTED;
  if ((double)rows * *st + (double)heads * *sh > 9.0e18) return SSBA_ERR_SHAPE;
  return SSBA_OK;
}

ssba_status check_query(const ssba_cache* c, const ssba_cache_batch* b, const ssba_cache_query* q) {
  if (!q) return SSBA_ERR_ARG;
  if (q->heads < 1 || q->heads % c->kv_heads) return SSBA_ERR_SHAPE;
  if (q->heads > 65536) return SSBA_ERR_UNSUPPORTED;
  if (q->dtype != SSBA_DT_BF16 && q->dtype != SSBA_DT_F32) return SSBA_ERR_ARG;
  if (q->causal != 0 && q->causal != 1) return SSBA_ERR_ARG;
  if (!std::isfinite(q->softmax_scale * kLog2e)) return SSBA_ERR_ARG;
  if ((int64_t)(q->heads / c->kv_heads) * b->max_new > kMaxTokens) return SSBA_ERR_UNSUPPORTED;
  if (q->keep < 0) return SSBA_ERR_ARG;
  if (q->keep > kMaxPages) return SSBA_ERR_UNSUPPORTED;
  return SSBA_OK;
}

ssba_status check_select(const ssba_cache_query* q) {
  if (q->keep < 1 || q->first < 0 || q->last < 1 || (int64_t)q->first + q->last > q->keep) return SSBA_ERR_ARG;
  return SSBA_OK;
}

CacheView view(const ssba_cache* c, int layer) {
  CacheView v;
  std::memset(&v, 0, sizeof(v));
  const int64_t rows = (int64_t)c->pages * c->kv_heads * layer;
  v.page_log2 = ilog2(c->page);
  v.page_bytes = (int64_t)c->kv_heads * c->page * c->head_dim;
  v.k = static_cast<uint8_t*>(c->k) + rows * c->page * c->head_dim;
  v.v = static_cast<uint8_t*>(c->v) + rows * c->page * c->head_dim;
  v.scale = c->scale + rows * 2;
  v.kmean = static_cast<uint16_t*>(c->kmean) + rows * c->head_dim;
  v.pages = c->pages;
  v.kv_heads = c->kv_heads;
  v.head_dim = c->head_dim;
  return v;
}

BatchView view(const ssba_cache_batch* b) {
  BatchView v;
  v.table = b->table;
  v.lens = b->lens;
  v.cu = b->cu;
  v.seqs = b->seqs;
  v.max_pages = b->max_pages;
  v.rows = b->rows;
  v.max_new = b->max_new;
  return v;
}

// About the longest sequence, by which work is split.
int64_t long_of(const ssba_cache* c, const ssba_cache_batch* b) {
  const int64_t most = (int64_t)b->max_pages * c->page;
  return b->max_len > 0 ? std::min<int64_t>(b->max_len, most) : most;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups that score, of one share of the pages each; in units of 256
// threads (512 in the tile form).
int64_t score_groups(const ssba_cache* c, const ssba_cache_batch* b, bool tile) {
  return tile ? (int64_t)b->seqs * c->kv_heads * ceil_div(b->max_new, 16) * 2 : (int64_t)b->rows * c->kv_heads;
}

// Pages to score fit a workgroup's LDS, or go through the scratch; 16 tokens
// share the pooled keys where sequences bring enough of them: with 8 of 16
// rows of a tile in use the matrix form needs half the loads.
ssba::SelectPlan plan_select(const ssba_cache* c, const ssba_cache_batch* b, const ssba_cache_query* q) {
  ssba::SelectPlan p;
  const bool tile = b->max_new >= 8;
  p.scored = b->max_pages > q->keep;
  p.chunks = 1;
  if (b->max_pages <= ssba::kSelectInLds) {
    p.kind = tile ? ssba::kSelectTile : ssba::kSelectRow;
  } else {
    p.kind = tile ? ssba::kSelectTileLong : ssba::kSelectRowLong;
    // A workgroup takes 64 pages at a time; 8 times as many for a tile, whose queries take longer to load.  Shares are
    // no more than a launch can have.
    const int64_t most = ssba::kMaxGroups256 / std::max<int64_t>(1, score_groups(c, b, tile));
    p.chunks = (int)std::min<int64_t>(ceil_div(ceil_div(long_of(c, b), c->page), ssba::kSelectPages * (tile ? 8 : 1)),
                                      std::max<int64_t>(1, std::min<int64_t>(most, 65535)));
  }
  return p;
}

size_t select_scratch(const ssba_cache* c, const ssba_cache_batch* b, const ssba_cache_query* q) {
  const ssba::SelectPlan p = plan_select(c, b, q);
  return p.scored && p.kind >= ssba::kSelectRowLong ? (size_t)8 * b->rows * c->kv_heads * b->max_pages : 0;
}

// Items are independent (sequence or row, kv head, column tile); one workgroup
// each, or several that share the item's keys where there are few items.
AttendPlan plan(const ssba_cache* c, const ssba_cache_batch* b, const ssba_cache_query* q, bool listed) {
  AttendPlan p;
  const int64_t group = q->heads / c->kv_heads;
  const int64_t cols = std::max<int64_t>(1, listed ? group : group * b->max_new);
  const bool f32 = q->dtype == SSBA_DT_F32;
  const int64_t keys = listed ? std::min<int64_t>((int64_t)q->keep * c->page, long_of(c, b)) : long_of(c, b);
  p.splits = p.tiles = 1;
  p.threads = 256;
  if (listed) {
    p.col_tiles = (int)ceil_div(cols, 16);
    const int64_t items = (int64_t)b->rows * c->kv_heads * p.col_tiles;
    // A wave each from 2 waves a SIMD on (2048 items of 2048 keys, D 128: 49 us, in 4 waves each 58; 1024: 34.7, 34.4).
    p.kind = items >= 2048 ? ssba::kAttendRows : ssba::kAttendRow;
    p.items = p.kind == ssba::kAttendRows ? ceil_div(b->rows, 4) * c->kv_heads * p.col_tiles : items;
  } else {
    // As many columns to a workgroup as there are, up to 256 (fp32: 32): its waves read the keys once for all.
    p.kind = ssba::kAttendSeq;
    while (p.tiles < (f32 ? 2 : 16) && cols > 16 * p.tiles) p.tiles *= 2;
    if (p.tiles >= 4) p.threads = 512;
    p.col_tiles = (int)ceil_div(cols, 16 * p.tiles);
    p.items = (int64_t)b->seqs * c->kv_heads * p.col_tiles;
  }
  const int64_t items = std::max<int64_t>(p.items, 1);
  if (p.tiles >= 4) {
    // One workgroup fills a CU.  Parts of at least 256 keys, as many as take the least time by these measured costs
    // in us: each round over the 256 CUs its beginning and end and its keys, the joining launch itself and its bytes
    // (written and read).  100 new tokens of 16 sequences, 16 heads on 4, D 64: of 600 tokens 22 us whole, 30 in two
    // parts; of 2000 48 us whole, 42 in two.
    const double d = c->head_dim, round = 3 + p.tiles * d / 400, key = p.tiles * (8e-4 + 6e-6 * d);
    const double column_bytes = 2.0 * 16 * p.tiles * d * 4;
    double best = ceil_div(items, 256) * (round + key * keys);
    for (int s = 2; s <= 256 && s * 256 <= keys && s * items <= 1024; ++s) {
      const double cost = ceil_div(items * s, 256) * (round + key * keys / s) + 3.5 + items * s * column_bytes / 3.6e6;
      if (cost < best * 0.98) {
        best = cost;
        p.splits = s;
      }
    }
  } else if (p.kind != ssba::kAttendRows && (p.tiles == 1 || !f32) && keys > 256 && items <= 256 &&
             keys <= (items >= (f32 ? 256 : 128) ? 4096 : 2048)) {
    // 8 waves of one workgroup instead of parts that a second launch joins: where such workgroups fill half the
    // chip (208 items of 2048 listed keys, D 128: 20.3 us, in 3 parts 21.5 + 4.0; 160 items of 4000: 28.7 us, in 4
    // parts 29.8 + 4.2), or an item is short (D 128, launches on the device, then calls from Python: 4 items of 1024
    // keys 7.8 and 13.6 us, in parts 8.1 and 18; 64 of 1536 11.3 and 13.6, 11.8 and 18; 4 of 2048 11.5 and 13.5, 8.8
    // and 18).  Few long ones need more CUs (4 items of 4096 keys 18.6 and 18.8 us, in parts 8.1 and 18), and long
    // ragged ones more parts (40 sequences of up to 8000 keys: 57 us, in parts 53).  fp32 (more vector work), D
    // 128: 256 items of 4000 keys 52 us, in parts 58; 128 of 2000 17.8, 20.1; 128 ragged ones of up to 2999 21.0, 20.2.
    // 32 columns, D 128: 64 items of 600 keys 9.9 us, in parts 11.9.
    p.threads = 512;
  } else if (p.kind != ssba::kAttendRows) {
    // 4 waves of at least 2 steps of 32 keys each, up to about 512 workgroups: more of them fill the chip more
    // evenly but begin and end more often (one sequence of 131072 keys, 4 heads, D 128: 512 33 us, 1024 41 us;
    // 64 ragged sequences: 128 and 131 us).
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(256, keys / 256));
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(most, ceil_div(512, items)));
  }
  return p;
}

// Columns of every part of a split launch.
size_t part_columns(const AttendPlan& p) { return p.splits == 1 ? 0 : (size_t)p.items * p.splits * p.tiles * 16; }

size_t attend_scratch(const ssba_cache* c, const AttendPlan& p) {
  return part_columns(p) * (c->head_dim + 2) * sizeof(float);
}

bool too_many(int64_t groups) { return groups > ssba::kMaxGroups256; }

}  // namespace

extern "C" {

ssba_status ssba_cache_append(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b, int32_t dtype,
                              const void* k, const void* v, int64_t stride_t, int64_t stride_h, void* stream) {
  ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if ((st = check_batch(c, b)) != SSBA_OK) return st;
  if (layer < 0 || layer >= c->layers) return SSBA_ERR_ARG;
  if ((st = strides_of(dtype, c->kv_heads, c->head_dim, b->rows, &stride_t, &stride_h)) != SSBA_OK) return st;
  if ((st = check_arrays(c)) != SSBA_OK || (st = check_batch_arrays(b)) != SSBA_OK) return st;
  if (b->rows == 0 || b->max_new == 0) return SSBA_OK;
  const size_t al = dtype == SSBA_DT_BF16 ? 16 : 4;
  if (!k || !v || !aligned(k, al) || !aligned(v, al)) return SSBA_ERR_ARG;
  ssba::AppendArgs a;
  a.c = view(c, layer);
  a.b = view(b);
  a.k = k;
  a.v = v;
  a.st = stride_t;
  a.sh = stride_h;
  a.slots = (int)std::min<int64_t>(((int64_t)b->max_new + 2 * c->page - 2) / c->page, b->max_pages);
  if (too_many((int64_t)b->seqs * a.slots * c->kv_heads)) return SSBA_ERR_UNSUPPORTED;
  return ssba::launch_cache_append(a, dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? SSBA_OK : SSBA_ERR_HIP;
}

ssba_status ssba_cache_select_workspace_size(const ssba_cache* c, const ssba_cache_batch* b,
                                             const ssba_cache_query* q, size_t* scratch_bytes) {
  ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if ((st = check_batch(c, b)) != SSBA_OK || (st = check_query(c, b, q)) != SSBA_OK || (st = check_select(q)) != SSBA_OK)
    return st;
  if (scratch_bytes) *scratch_bytes = select_scratch(c, b, q);
  return SSBA_OK;
}

ssba_status ssba_cache_select(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b,
                              const ssba_cache_query* q, const void* query, int32_t* lists, size_t lists_bytes,
                              void* scratch, size_t scratch_bytes, void* stream) {
  ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if ((st = check_batch(c, b)) != SSBA_OK || (st = check_query(c, b, q)) != SSBA_OK || (st = check_select(q)) != SSBA_OK)
    return st;
  if (layer < 0 || layer >= c->layers) return SSBA_ERR_ARG;
  ssba::SelectArgs a;
  a.st = q->q_stride_t;
  a.sh = q->q_stride_h;
  if ((st = strides_of(q->dtype, q->heads, c->head_dim, b->rows, &a.st, &a.sh)) != SSBA_OK) return st;
  if ((st = check_arrays(c)) != SSBA_OK || (st = check_batch_arrays(b)) != SSBA_OK) return st;
  if (b->rows == 0 || b->max_new == 0) return SSBA_OK;
  const size_t need = select_scratch(c, b, q);
  if (!query || !lists || !aligned(query, q->dtype == SSBA_DT_BF16 ? 16 : 4) || !aligned(lists, 4)) return SSBA_ERR_ARG;
  if (need && (!scratch || !aligned(scratch, 16))) return SSBA_ERR_ARG;
  if (lists_bytes < (size_t)4 * b->rows * c->kv_heads * (1 + (size_t)q->keep) || scratch_bytes < need)
    return SSBA_ERR_WORKSPACE;
  a.c = view(c, layer);
  a.b = view(b);
  a.q = query;
  a.lists = lists;
  a.keys = static_cast<uint64_t*>(scratch);
  a.group = q->heads / c->kv_heads;
  a.causal = q->causal;
  a.keep = q->keep;
  a.first = q->first;
  a.last = q->last;
  a.tiles = (int)ceil_div(b->max_new, 16);
  const ssba::SelectPlan p = plan_select(c, b, q);
  // 1024 threads at most rank a row, 512 score one where its keys stay in the LDS.
  const bool tile = p.kind == ssba::kSelectTile || p.kind == ssba::kSelectTileLong;
  if (too_many((int64_t)b->rows * c->kv_heads * 4) || too_many(score_groups(c, b, tile) * p.chunks))
    return SSBA_ERR_UNSUPPORTED;
  return ssba::launch_cache_select(a, p, q->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? SSBA_OK
                                                                                                   : SSBA_ERR_HIP;
}

ssba_status ssba_cache_attend_workspace_size(const ssba_cache* c, const ssba_cache_batch* b,
                                             const ssba_cache_query* q, int32_t with_lists, size_t* scratch_bytes) {
  ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if ((st = check_batch(c, b)) != SSBA_OK || (st = check_query(c, b, q)) != SSBA_OK) return st;
  if (with_lists && q->keep < 1) return SSBA_ERR_ARG;
  if (scratch_bytes) *scratch_bytes = attend_scratch(c, plan(c, b, q, with_lists != 0));
  return SSBA_OK;
}

ssba_status ssba_cache_attend(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b,
                              const ssba_cache_query* q, const void* query, const int32_t* lists, size_t lists_bytes,
                              void* o, void* scratch, size_t scratch_bytes, void* stream) {
  ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if ((st = check_batch(c, b)) != SSBA_OK || (st = check_query(c, b, q)) != SSBA_OK) return st;
  if (layer < 0 || layer >= c->layers) return SSBA_ERR_ARG;
  if (lists && q->keep < 1) return SSBA_ERR_ARG;
  AttendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.q_st = q->q_stride_t;
  a.q_sh = q->q_stride_h;
  a.o_st = q->o_stride_t;
  a.o_sh = q->o_stride_h;
  if ((st = strides_of(q->dtype, q->heads, c->head_dim, b->rows, &a.q_st, &a.q_sh)) != SSBA_OK) return st;
  if ((st = strides_of(q->dtype, q->heads, c->head_dim, b->rows, &a.o_st, &a.o_sh)) != SSBA_OK) return st;
  if ((st = check_arrays(c)) != SSBA_OK || (st = check_batch_arrays(b)) != SSBA_OK) return st;
  if (b->rows == 0 || b->max_new == 0) return SSBA_OK;
  const size_t al = q->dtype == SSBA_DT_BF16 ? 16 : 4;
  if (!query || !o || !aligned(query, al) || !aligned(o, al) || !aligned(lists, 4)) return SSBA_ERR_ARG;
  const AttendPlan p = plan(c, b, q, lists != nullptr);
  const size_t need = attend_scratch(c, p);
  if (need && (!scratch || !aligned(scratch, 16))) return SSBA_ERR_ARG;
  if (scratch_bytes < need || (lists && lists_bytes < (size_t)4 * b->rows * c->kv_heads * (1 + (size_t)q->keep)))
    return SSBA_ERR_WORKSPACE;
  if (too_many(p.items * p.splits * 4) || too_many(p.items * p.tiles * 4)) return SSBA_ERR_UNSUPPORTED;
  a.c = view(c, layer);
  a.b = view(b);
  a.q = query;
  a.o = o;
  a.lists = lists;
  a.part = static_cast<float*>(scratch);
  a.part_ml = need ? a.part + part_columns(p) * c->head_dim : nullptr;
  const float scale = q->softmax_scale > 0.f ? q->softmax_scale : 1.0f / std::sqrt((float)c->head_dim);
  a.scale_log2 = scale * kLog2e;
  a.group = q->heads / c->kv_heads;
  a.causal = q->causal;
  a.keep = q->keep;
  a.col_tiles = p.col_tiles;
  a.splits = p.splits;
  return ssba::launch_cache_attend(a, p, q->dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? SSBA_OK
                                                                                                   : SSBA_ERR_HIP;
}

}  // extern "C"

namespace {

ssba_status check_pages(const ssba_cache* c, const ssba_pages* p) {
  const ssba_status st = check_shape(c);
  if (st != SSBA_OK) return st;
  if (!p) return SSBA_ERR_ARG;
  if (p->rows < 1 || p->max_pages < 1) return SSBA_ERR_SHAPE;
  if ((int64_t)p->rows * p->max_pages >= ((int64_t)1 << 31) || (int64_t)p->max_pages * c->page > kMaxTokens)
    return SSBA_ERR_UNSUPPORTED;
  return SSBA_OK;
}

// int32 elements: the larger of what each call keeps (see ssba_cache_pages.hip).
size_t pages_scratch(const ssba_cache* c, const ssba_pages* p, int64_t n) {
  const size_t reserve = (size_t)p->rows * p->max_pages + p->rows;
  const size_t fork = 4 + (size_t)3 * n + (size_t)2 * p->rows;
  const size_t compact = 4 + (size_t)3 * c->pages;
  return 4 * std::max(reserve, std::max(fork, compact));
}

ssba_status pages_args(const ssba_cache* c, const ssba_pages* p, int32_t n, const void* x, const void* y,
                       int32_t* info, void* scratch, size_t scratch_bytes, ssba::PagesArgs* a) {
  const ssba_status st = check_pages(c, p);
  if (st != SSBA_OK) return st;
  if (n < 0) return SSBA_ERR_SHAPE;
  if (n > kMaxPages || (int64_t)n * p->max_pages >= ((int64_t)1 << 31)) return SSBA_ERR_UNSUPPORTED;
  if (!p->table || !p->lens || !p->refs || !info || !scratch || (n > 0 && (!x || !y))) return SSBA_ERR_ARG;
  if (!aligned(p->table, 4) || !aligned(p->lens, 4) || !aligned(p->refs, 4) || !aligned(info, 4) ||
      !aligned(x, 4) || !aligned(y, 4) || !aligned(scratch, 16))
    return SSBA_ERR_ARG;
  if (scratch_bytes < pages_scratch(c, p, n)) return SSBA_ERR_WORKSPACE;
  std::memset(a, 0, sizeof(*a));
  a->rows = p->rows;
  a->max_pages = p->max_pages;
  a->pages = c->pages;
  a->page_log2 = ilog2(c->page);
  a->table = p->table;
  a->lens = p->lens;
  a->refs = p->refs;
  a->info = info;
  a->scratch = static_cast<int32_t*>(scratch);
  a->src = static_cast<const int32_t*>(x);
  a->dst = static_cast<const int32_t*>(y);
  a->n = n;
  return SSBA_OK;
}

ssba::CopyArgs copy_args(const ssba_cache* from, const ssba_cache* to) {
  ssba::CopyArgs a;
  std::memset(&a, 0, sizeof(a));
  const void* f[4] = {from->k, from->v, from->scale, from->kmean};
  void* t[4] = {to->k, to->v, to->scale, to->kmean};
  const int64_t codes = (int64_t)from->kv_heads * from->page * from->head_dim;
  const int64_t bytes[4] = {codes, codes, (int64_t)from->kv_heads * 8, (int64_t)from->kv_heads * from->head_dim * 2};
  for (int i = 0; i < 4; ++i) {
    a.from[i] = static_cast<const char*>(f[i]);
    a.to[i] = static_cast<char*>(t[i]);
    a.bytes[i] = bytes[i];
    a.from_layer[i] = bytes[i] * from->pages;
    a.to_layer[i] = bytes[i] * to->pages;
  }
  a.layers = from->layers;
  a.from_pages = from->pages;
  a.to_pages = to->pages;
  return a;
}

ssba_status status_of(hipError_t e) { return e == hipSuccess ? SSBA_OK : SSBA_ERR_HIP; }

}  // namespace

extern "C" {

ssba_status ssba_pages_workspace_size(const ssba_cache* c, const ssba_pages* p, int32_t n, size_t* scratch_bytes) {
  const ssba_status st = check_pages(c, p);
  if (st != SSBA_OK) return st;
  if (n < 0) return SSBA_ERR_SHAPE;
  if (scratch_bytes) *scratch_bytes = pages_scratch(c, p, n);
  return SSBA_OK;
}

ssba_status ssba_pages_reserve(const ssba_cache* c, const ssba_pages* p, int32_t* info, void* scratch,
                               size_t scratch_bytes, void* stream) {
  ssba::PagesArgs a;
  const ssba_status st = pages_args(c, p, 0, nullptr, nullptr, info, scratch, scratch_bytes, &a);
  return st != SSBA_OK ? st : status_of(ssba::launch_pages_reserve(a, static_cast<hipStream_t>(stream)));
}

ssba_status ssba_pages_fork(const ssba_cache* c, const ssba_pages* p, int32_t n, const int32_t* src,
                            const int32_t* dst, int32_t* info, void* scratch, size_t scratch_bytes, void* stream) {
  ssba::PagesArgs a;
  ssba_status st = pages_args(c, p, n, src, dst, info, scratch, scratch_bytes, &a);
  if (st != SSBA_OK || (st = check_arrays(c)) != SSBA_OK) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ssba::launch_pages_fork(a, hs) != hipSuccess) return SSBA_ERR_HIP;
  if (n == 0) return SSBA_OK;
  ssba::CopyArgs m = copy_args(c, c);
  m.count = a.scratch;
  m.src = a.scratch + 4;
  m.dst = m.src + n;
  m.n = n;
  return status_of(ssba::launch_pages_copy(m, hs));
}

ssba_status ssba_pages_release(const ssba_cache* c, const ssba_pages* p, int32_t n, const int32_t* row, int32_t* info,
                               void* scratch, size_t scratch_bytes, void* stream) {
  ssba::PagesArgs a;
  const ssba_status st = pages_args(c, p, n, row, row, info, scratch, scratch_bytes, &a);
  return st != SSBA_OK ? st : status_of(ssba::launch_pages_release(a, static_cast<hipStream_t>(stream)));
}

ssba_status ssba_pages_compact(const ssba_cache* c, const ssba_pages* p, int32_t* table_out, int32_t* refs_out,
                               int32_t* info, void* scratch, size_t scratch_bytes, void* stream) {
  ssba::PagesArgs a;
  ssba_status st = pages_args(c, p, 0, nullptr, nullptr, info, scratch, scratch_bytes, &a);
  if (st != SSBA_OK || (st = check_arrays(c)) != SSBA_OK) return st;
  if (!table_out || !refs_out || !aligned(table_out, 4) || !aligned(refs_out, 4)) return SSBA_ERR_ARG;
  a.table_out = table_out;
  a.refs_out = refs_out;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ssba::launch_pages_compact(a, hs) != hipSuccess) return SSBA_ERR_HIP;
  ssba::CopyArgs m = copy_args(c, c);
  m.count = a.scratch;
  m.src = a.scratch + 4;
  m.dst = m.src + c->pages;
  m.n = std::max(1, c->pages / 2);   // at most half of the pages move
  m.map = m.dst + c->pages;
  m.table = p->table;
  m.table_out = table_out;
  m.entries = (int64_t)p->rows * p->max_pages;
  return status_of(ssba::launch_pages_copy(m, hs));
}

ssba_status ssba_pages_copy(const ssba_cache* from, const ssba_cache* to, int32_t n, const int32_t* src,
                            const int32_t* dst, void* stream) {
  ssba_status st = check_shape(from);
  if (st != SSBA_OK || (st = check_shape(to)) != SSBA_OK) return st;
  if (from->layers != to->layers || from->kv_heads != to->kv_heads || from->head_dim != to->head_dim ||
      from->page != to->page || n < 0)
    return SSBA_ERR_SHAPE;
  if ((st = check_arrays(from)) != SSBA_OK || (st = check_arrays(to)) != SSBA_OK) return st;
  if (n == 0) return SSBA_OK;
  if (!src || !dst || !aligned(src, 4) || !aligned(dst, 4)) return SSBA_ERR_ARG;
  ssba::CopyArgs a = copy_args(from, to);
  a.src = src;
  a.dst = dst;
  a.n = n;
  return status_of(ssba::launch_pages_copy(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
