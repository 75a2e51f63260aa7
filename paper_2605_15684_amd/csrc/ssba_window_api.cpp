// C ABI of the windowed attention: argument checks, workspace size and launch
// plans.  See include/ssba_window.h for the contract.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "ssba_common.h"
#include "ssba_window_common.h"

namespace {

using ssba::kWindowRows;
using ssba::Strides;
using ssba::WindowArgs;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kMostParts = (int64_t)256 << 20;   // bytes of the parts of sink tiles

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

ssba_status check(const ssba_window* w) {
  if (!w) return SSBA_ERR_ARG;
  if (w->batch < 0 || w->seq < 0 || w->heads < 1 || w->kv_heads < 1 || w->heads % w->kv_heads) return SSBA_ERR_SHAPE;
  if (w->head_dim != 64 && w->head_dim != 128) return SSBA_ERR_UNSUPPORTED;
  if (w->dtype != SSBA_DT_BF16 && w->dtype != SSBA_DT_F32) return SSBA_ERR_ARG;
  if (w->window < 1 || w->sinks < 0 || w->max_len < 0) return SSBA_ERR_ARG;
  if (!std::isfinite(w->softmax_scale * kLog2e)) return SSBA_ERR_ARG;
  if (w->heads > 65536 || w->batch > (1 << 24) || w->seq > (1 << 30)) return SSBA_ERR_UNSUPPORTED;
  if (w->seqs < 0 || w->seqs > 65535) return SSBA_ERR_UNSUPPORTED;
  if (w->seqs ? w->batch != 1 : w->cu != nullptr) return SSBA_ERR_SHAPE;
  return SSBA_OK;
}

// Element strides of a [batch][heads][seq][D] array; all 0: contiguous.  `out`: rows that are written must not overlap.
ssba_status strides_of(const ssba_window* w, int heads, bool out, const ssba_strides& from, Strides* s) {
  s->b = from.b;
  s->h = from.h;
  s->t = from.t;
  if (s->b == 0 && s->h == 0 && s->t == 0) {
    s->t = w->head_dim;
    s->h = (int64_t)w->seq * s->t;
    s->b = heads * s->h;
  }
  if (s->b < 0 || s->h < 0 || s->t < 0) return SSBA_ERR_SHAPE;
  if ((w->seq > 1 && s->t < w->head_dim) || (w->seq > 0 && heads > 1 && s->h < w->head_dim) ||
      (out && w->seq > 0 && w->batch > 1 && s->b < w->head_dim))
    return SSBA_ERR_SHAPE;
  if ((s->b | s->h | s->t) & (w->dtype == SSBA_DT_BF16 ? 7 : 3)) return SSBA_ERR_UNSUPPORTED;
  if (s->t > (1 << 20)) return SSBA_ERR_UNSUPPORTED;
  if ((double)w->batch * s->b + (double)heads * s->h + (double)w->seq * s->t > 2.0e18) return SSBA_ERR_SHAPE;
  return SSBA_OK;
}

// The launch plan: everything that goes by the descriptor alone.
ssba_status plan(const ssba_window* w, WindowArgs* a) {
  std::memset(a, 0, sizeof(*a));
  ssba_status st;
  if ((st = strides_of(w, w->heads, false, w->q, &a->sq)) != SSBA_OK ||
      (st = strides_of(w, w->kv_heads, false, w->k, &a->sk)) != SSBA_OK ||
      (st = strides_of(w, w->kv_heads, false, w->v, &a->sv)) != SSBA_OK ||
      (st = strides_of(w, w->heads, true, w->o, &a->so)) != SSBA_OK)
    return st;
  a->cu = w->cu;
  a->batch = w->batch;
  a->seq = w->seq;
  a->heads = w->heads;
  a->kv_heads = w->kv_heads;
  a->group = w->heads / w->kv_heads;
  a->window = std::max(1, std::min(w->window, w->seq));   // no token sees further back
  a->sinks = std::min(w->sinks, w->seq);
  a->seqs = w->seqs;
  a->scale = w->softmax_scale > 0.f ? w->softmax_scale : 1.0f / std::sqrt((float)w->head_dim);
  a->scale_log2 = a->scale * kLog2e;
  a->slots = w->seqs ? w->seq / kWindowRows + w->seqs + 1 : (int)ceil_div(w->seq, kWindowRows);
  if ((double)w->batch * w->heads * a->slots > (double)ssba::kMaxGroups256) return SSBA_ERR_UNSUPPORTED;
  // Tiles of every head in turn, long ones first, where the heads go evenly to the XCDs or tiles differ much in length;
  // else the tiles of a head together.
  const int64_t units = (int64_t)w->batch * w->kv_heads;
  const int64_t longest = w->seqs && w->max_len ? std::min(w->max_len, w->seq) : w->seq;
  a->spread = units % 8 == 0 || (int64_t)w->window * 4 > longest;
  // Tiles of sink keys are seen by all later queries: cut into chunks of what the window leaves other tiles, but of at
  // least 1024 queries, and not into more than about 64 a head.  Behind narrow windows these chunks are the longest of the
  // launch (8192 rows, D 128, backward with 4 sinks and none: bf16, 8 heads, window 16 85.5 and 53.0 us, 128 88.2 and
  // 59.6, 512 129 and 99; 16 heads on 4, window 64 158 and 94; fp32 752 and 274).
  a->sink_tiles = (int)ceil_div(a->sinks, kWindowRows);
  const int64_t chunk = std::max<int64_t>({1024, (int64_t)w->window + kWindowRows, (int64_t)w->seq * a->sink_tiles / 64});
  a->chunk = (int)std::min<int64_t>(ceil_div(chunk, kWindowRows) * kWindowRows, (int64_t)1 << 30);
  if (a->sinks && longest > a->chunk) {
    const int64_t slots = w->seqs ? w->seq / a->chunk + w->seqs + 1 : ceil_div(w->seq, a->chunk);
    const double bytes = (double)units * a->sink_tiles * slots * 2 * kWindowRows * w->head_dim * 4;
    if (bytes <= kMostParts) a->chunk_slots = (int)slots;
  }
  const int64_t cut = (int64_t)a->sink_tiles * a->chunk_slots;
  // The heads of a group are shared evenly by several workgroups where those of whole tiles do not fill the chip (two a
  // CU; fp32: one), as far as their parts stay within that size.
  const int64_t tiles = std::max<int64_t>(1, units * (a->slots + cut)), room = w->dtype == SSBA_DT_F32 ? 256 : 512;
  const int64_t most = kMostParts / (tiles * 2 * kWindowRows * w->head_dim * 4);
  a->head_parts = 1;
  for (int n = 2; n <= a->group && n <= most && tiles * a->head_parts < room; ++n)
    if (a->group % n == 0) a->head_parts = n;
  // Then the queries, in shares of at least 128 (fp32) or 256 (bf16, D 128), whose tiles take long enough to be worth
  // their parts; the join walks a tile's parts in turn, so at most 16.  Backward, one share against several: 1024 rows, 8
  // heads, window 256, fp32 D 128 208 to 128 us, D 64 104 to 76 (shares of 64: 117, 72); 16 heads on 4, window 1024, bf16 D 128 80 to 71; but
  // D 64 49 to 52.  8 heads on 2, 512 rows, fp32 D 64: 20 parts 68, 32 parts 80.
  a->query_parts = 1;
  const int64_t least = w->dtype == SSBA_DT_F32 ? kWindowRows : w->head_dim == 128 ? 256 : 0;
  if (least) {
    const int64_t queries = std::min<int64_t>((int64_t)a->window + kWindowRows, longest);
    const int64_t n = std::min<int64_t>({room / (tiles * a->head_parts), queries / least, std::min<int64_t>(most, 16) / a->head_parts});
    a->query_parts = (int)std::max<int64_t>(1, n);
  }
  const int64_t shares = (int64_t)a->head_parts * a->query_parts;
  // The key side's launch, and the join's of 8 workgroups a part.
  const int64_t kept = cut + (shares > 1 ? a->slots : 0);
  if ((double)units * (a->slots + cut) * shares > (double)ssba::kMaxGroups256 ||
      (double)units * kept * 8 > (double)ssba::kMaxGroups256)
    return SSBA_ERR_UNSUPPORTED;
  return SSBA_OK;
}

size_t part_bytes(const ssba_window* w, const WindowArgs& a) {
  const size_t shares = (size_t)a.head_parts * a.query_parts;
  const size_t kept = (size_t)a.sink_tiles * a.chunk_slots + (shares > 1 ? a.slots : 0);
  return (size_t)w->batch * w->kv_heads * kept * shares * 2 * kWindowRows * w->head_dim * 4;
}

size_t row_bytes(const ssba_window* w) { return ceil_div((int64_t)w->batch * w->heads * w->seq * 4, 256) * 256; }

bool empty(const ssba_window* w) { return w->batch == 0 || w->seq == 0; }

}  // namespace

extern "C" {

ssba_status ssba_window_forward(const ssba_window* w, const void* q, const void* k, const void* v, void* o, float* lse,
                                void* hip_stream) {
  ssba_status st = check(w);
  if (st != SSBA_OK) return st;
  WindowArgs a;
  if ((st = plan(w, &a)) != SSBA_OK) return st;
  if (empty(w)) return SSBA_OK;
  if (!q || !k || !v || !o || (w->seqs && !w->cu)) return SSBA_ERR_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(w->cu, 4))
    return SSBA_ERR_ARG;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = lse;
  return ssba::launch_window_forward(a, w->head_dim, w->dtype, static_cast<hipStream_t>(hip_stream)) == hipSuccess
             ? SSBA_OK
             : SSBA_ERR_HIP;
}

ssba_status ssba_window_backward_workspace_size(const ssba_window* w, size_t* scratch_bytes) {
  ssba_status st = check(w);
  if (st != SSBA_OK) return st;
  WindowArgs a;
  if ((st = plan(w, &a)) != SSBA_OK) return st;
  if (scratch_bytes) *scratch_bytes = empty(w) ? 0 : 2 * row_bytes(w) + part_bytes(w, a);
  return SSBA_OK;
}

ssba_status ssba_window_backward(const ssba_window* w, const ssba_window_grads* g, const void* q, const void* k,
                                 const void* v, const void* o, const void* dout, const float* lse, void* dq, void* dk,
                                 void* dv, void* scratch, size_t scratch_bytes, void* hip_stream) {
  ssba_status st = check(w);
  if (st != SSBA_OK) return st;
  if (!g) return SSBA_ERR_ARG;
  WindowArgs a;
  if ((st = plan(w, &a)) != SSBA_OK) return st;
  if ((st = strides_of(w, w->heads, false, g->do_, &a.sdo)) != SSBA_OK ||
      (st = strides_of(w, w->heads, true, g->dq, &a.sdq)) != SSBA_OK ||
      (st = strides_of(w, w->kv_heads, true, g->dk, &a.sdk)) != SSBA_OK ||
      (st = strides_of(w, w->kv_heads, true, g->dv, &a.sdv)) != SSBA_OK)
    return st;
  if (empty(w)) return SSBA_OK;
  if (!q || !k || !v || !o || !dout || !lse || !dq || !dk || !dv || !scratch || (w->seqs && !w->cu)) return SSBA_ERR_ARG;
  for (const void* p : {q, k, v, o, dout, static_cast<const void*>(dq), static_cast<const void*>(dk),
                        static_cast<const void*>(dv), static_cast<const void*>(scratch)})
    if (!aligned(p, 16)) return SSBA_ERR_ARG;
  if (!aligned(lse, 4) || !aligned(w->cu, 4)) return SSBA_ERR_ARG;
  if (scratch_bytes < 2 * row_bytes(w) + part_bytes(w, a)) return SSBA_ERR_WORKSPACE;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = const_cast<void*>(o);
  a.dout = dout;
  a.lse = const_cast<float*>(lse);
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.lse2 = static_cast<float*>(scratch);
  a.ndelta = a.lse2 + row_bytes(w) / 4;
  a.part = a.ndelta + row_bytes(w) / 4;
  return ssba::launch_window_backward(a, w->head_dim, w->dtype, static_cast<hipStream_t>(hip_stream)) == hipSuccess
             ? SSBA_OK
             : SSBA_ERR_HIP;
}

}  // extern "C"
