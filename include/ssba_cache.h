/*
 * ssba_cache.h -- C ABI of the paged 8-bit key/value cache for AMD Instinct
 * MI355X (gfx950): generation with the keys and values of earlier calls kept,
 * in the same library as ssba.h.
 *
 * A cache holds the keys and values of sequences in pages of `page` tokens, in
 * e4m3 (1 byte a value) with one scale per page and kv head.  A page table
 * names the pages of each sequence in order.  Query heads h * G .. h * G + G-1
 * (G = heads / kv_heads) read kv head h.
 *
 *   append   quantises new keys and values into the pages
 *   select   the top-k gate of ssba.h for single queries: a cheap score of
 *            each page (pooled keys) keeps `keep` pages per token and kv head
 *   attend   attention of new tokens over the whole sequence or the selected
 *            pages
 *   pages    reserve, fork, release, copy and compact
 *
 * Arrays of a cache (device memory, owned by the caller):
 *   k, v   e4m3 [layers][pages][kv_heads][page * D], 16-byte aligned.  The
 *          codes of 16 tokens lie together in the operand order of the matrix
 *          instructions: with token t = 16 T + r and channel c, the byte
 *            K: 16 D T + 1024 (c/64) + 256 (c%64 / 16) + 16 r + c%16
 *            V: 16 D T + 1024 (c/64) + 256 (r/4) + 16 (c%16) + 4 (c%64 / 16) + r%4
 *          of its page (16-byte loads of a wave are 1024 consecutive bytes).
 *   scale  fp32 [layers][pages][kv_heads][2], 8-byte aligned: a key is
 *          scale[0] * code, a value scale[1] * code; 2^-64 to 2^120 (append
 *          writes powers of two).
 *   kmean  bf16 [layers][pages][kv_heads][D], 16-byte aligned: the mean of the
 *          keys of a complete page (select reads it; attend does not).
 * Nothing has to be initialised: slots behind a sequence's end are never used,
 * whatever they hold.
 *
 * Sequences of a call (ssba_cache_batch; device arrays of int32):
 *   table  [seqs][max_pages]: page numbers; an entry outside 0..pages-1 is a
 *          page that is not there (its tokens are neither written nor seen)
 *   lens   [seqs]: tokens a sequence holds, this call's new ones included
 *   cu     [seqs + 1]: rows cu[s] .. cu[s+1]-1 of the packed arrays (K, V, Q,
 *          O) are the new tokens of sequence s, the last cu[s+1]-cu[s] that it
 *          holds; 0 rows: an idle sequence.  cu must not decrease.
 * Rows of the packed arrays that belong to no sequence are not written, and no
 * result depends on what they hold (select may read them).  The values are read
 * on the device, so a captured call replays with new lengths; whatever they are,
 * no access leaves the arrays.  Tokens of a sequence past max_pages * page are
 * neither written nor seen, rows past `rows` are not the sequence's; a sequence
 * that holds fewer tokens than it has new rows is not appended, its earliest
 * rows see nothing.
 *
 * Ownership, streams and errors as in ssba.h: the caller owns every buffer,
 * calls are asynchronous on `hip_stream`, checks come before any launch, and
 * nothing is allocated or kept between calls.  Calls that overlap in time must
 * not share a scratch buffer.
 */
#ifndef SSBA_CACHE_H_
#define SSBA_CACHE_H_

#include "ssba.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ssba_cache {
  int32_t layers, pages;     /* 1 <= layers <= 65534, 1 <= pages <= 2^24          */
  int32_t kv_heads;          /* 1 .. 1024                                        */
  int32_t head_dim;          /* 64 or 128                                        */
  int32_t page;              /* tokens per page: 16, 32 or 64                    */
  void* k;
  void* v;
  float* scale;
  void* kmean;
} ssba_cache;

typedef struct ssba_cache_batch {
  int32_t seqs;              /* 1 .. 65535                                       */
  int32_t max_pages;         /* columns of the table; max_pages * page <= 2^30   */
  int32_t rows;              /* rows of the packed arrays (bounds every access)  */
  int32_t max_new;           /* at least the new tokens of any sequence          */
  int32_t max_len;           /* about the longest sequence (only how work is split goes by it); 0: max_pages * page */
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
} ssba_cache_batch;

/* Queries of ssba_cache_select and ssba_cache_attend. */
typedef struct ssba_cache_query {
  int32_t heads;             /* query heads, a multiple of kv_heads              */
  int32_t dtype;             /* ssba_dtype of Q and O                            */
  int32_t causal;            /* 1: a token sees itself and what is before it; 0: the whole sequence */
  int32_t keep;              /* pages per token and kv head, 1 .. 2^24 (0 without lists) */
  int32_t first, last;       /* select: leading and trailing pages always kept; first >= 0, last >= 1, first + last <= keep */
  float softmax_scale;       /* <= 0 selects 1 / sqrt(head_dim); at most 2^127   */
  int64_t q_stride_t, q_stride_h; /* element strides of Q [rows][heads][D]; both 0 = contiguous */
  int64_t o_stride_t, o_stride_h; /* the same of O                               */
} ssba_cache_query;

/* Quantises the new tokens' keys and values into the pages of `layer`.
 * K and V [rows][kv_heads][D] in `dtype` share the element strides (stride_t,
 * stride_h) (both 0 = contiguous); bf16: 16-byte aligned, strides multiples of
 * 8; fp32: 4-byte aligned.
 *   A page's scale is 2^e with the smallest e >= -64 that holds every finite
 * value put into it since its first token: |x| <= 448 * 2^e.  A value is held
 * as code = e4m3(x * 2^-e), to nearest, ties to even; +-inf as +-448, NaN as
 * NaN.  In a page that holds older tokens 2^e also reaches the scale s that it
 * has, which need not be a power of two; where s is not 2^e, the older codes are
 * restated as e4m3(code * (s * 2^-e)), the product in fp32.  When the last
 * token of a page comes, kmean = bf16(2^e * sum(codes) / page).  The result does
 * not depend on atomics or on the order of workgroups.  Pages that several rows
 * share (ssba_pages_fork) must be complete; two sequences of a call must not append
 * to one page. */
ssba_status ssba_cache_append(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b, int32_t dtype,
                              const void* k, const void* v, int64_t stride_t, int64_t stride_h, void* hip_stream);

/* Device bytes of the scratch of ssba_cache_select for this cache, batch and
 * query: 0 for tables of up to 1152 pages or up to `keep`, else 8 * rows *
 * kv_heads * max_pages (4096 rows, 8 heads, 16384 pages: 4.3 GB). */
ssba_status ssba_cache_select_workspace_size(const ssba_cache* c, const ssba_cache_batch* b,
                                             const ssba_cache_query* q, size_t* scratch_bytes);

/* Selects `keep` pages for every new token and kv head.  A token at position p
 * (causal) has the pages 0 .. p / page; without causal every token has those
 * of the whole sequence.  If there are more than `keep`, the `first` leading
 * and the `last` trailing ones are kept and the other places go to the pages
 * between them with the largest score
 *   (sum over the query heads of the group, in order, of q) . kmean[page],
 * computed in 64 bits; equal scores keep the lower page, +0 == -0, NaN and
 * pages that are not there rank last.  `lists` int32 [rows][kv_heads][1 + keep]:
 * the count, page numbers of the sequence (columns of the table) ascending,
 * then -1.  Appending must come first: only complete pages are scored.
 * `scratch` 16-byte aligned (NULL where its size is 0). */
ssba_status ssba_cache_select(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b,
                              const ssba_cache_query* q, const void* query, int32_t* lists, size_t lists_bytes,
                              void* scratch, size_t scratch_bytes, void* hip_stream);

/* Device bytes of the scratch of ssba_cache_attend; `with_lists`: 1 if the call passes lists. */
ssba_status ssba_cache_attend_workspace_size(const ssba_cache* c, const ssba_cache_batch* b,
                                             const ssba_cache_query* q, int32_t with_lists, size_t* scratch_bytes);

/* Attention of every new token: o = softmax(scale * q K^T) V over the tokens
 * it sees (q->causal), of its whole sequence (lists NULL) or of the pages that
 * `lists` names for it and its kv head (as ssba_cache_select writes them;
 * counts are cut to 0 .. keep, entries that are no page of the sequence are
 * passed over, one that is named twice counts twice).  A token that sees
 * nothing gets zeros.
 *   bf16: Q as it is, codes exact, products and sums in fp32.  Probabilities
 * enter the value product with 16 bits (two bf16 terms) where G * max_new is 16
 * or less, with lists where rows * kv_heads * ceil(G / 16) is below 2048; else
 * with 11 (fp16, V's scale included; weights of less than 2^-22 of the largest
 * in steps of 2^-32 of it).  So a token's result depends on the rest of its
 * batch by such roundings, which are below that of O.  fp32: Q and the probabilities
 * as three bf16 terms each (24 bits), so products are those of fp32.  Sums are
 * formed before they are normalised: values beyond 2^90 may overflow.
 * bf16 Q and O 16-byte aligned with strides in multiples of 8, fp32 4-byte
 * aligned; `scratch` 16-byte aligned (NULL where its size is 0).  O must not
 * overlap Q. */
ssba_status ssba_cache_attend(const ssba_cache* c, int32_t layer, const ssba_cache_batch* b,
                              const ssba_cache_query* q, const void* query, const int32_t* lists, size_t lists_bytes,
                              void* o, void* scratch, size_t scratch_bytes, void* hip_stream);

/* ---- pages --------------------------------------------------------------
 * table [rows][max_pages], lens [rows], refs [pages]: how many table entries
 * name a page (0: free).  All are device int32 arrays updated by the calls in
 * stream order; entries outside 0..pages-1 mean "none".  Free pages are taken
 * lowest number first, so results are reproducible.  `info` int32[2] on the
 * device is written by each call.  Row numbers in `row`, `src`, `dst` that are
 * not in 0..rows-1 are passed over.  `scratch` (ssba_pages_workspace_size) is
 * 16-byte aligned. */
typedef struct ssba_pages {
  int32_t rows, max_pages;   /* 1 <= rows, rows * max_pages < 2^31               */
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
} ssba_pages;

/* Device bytes of the scratch of the calls below; n: the most rows or pairs of a call. */
ssba_status ssba_pages_workspace_size(const ssba_cache* c, const ssba_pages* p, int32_t n, size_t* scratch_bytes);

/* Gives every row s the pages that lens[s] tokens need: the entries below
 * ceil(lens[s] / page) that name none, in order of (row, entry), take the free
 * pages.  info = {entries served, entries left without a page}. */
ssba_status ssba_pages_reserve(const ssba_cache* c, const ssba_pages* p, int32_t* info, void* scratch,
                               size_t scratch_bytes, void* hip_stream);

/* Row dst[j] becomes a copy of row src[j]: it shares the complete pages and
 * gets a free page of its own, with the contents of every layer copied, for an
 * incomplete last one.  What row dst[j] named before is dropped without being
 * released.  A pair is passed over if its dst is another pair's (or its own)
 * src or an earlier pair's dst.  Where no page is free the last entry stays -1
 * and lens[dst] is cut to the complete pages.
 * info = {pairs forked, of them cut for lack of a page}. */
ssba_status ssba_pages_fork(const ssba_cache* c, const ssba_pages* p, int32_t n, const int32_t* src,
                            const int32_t* dst, int32_t* info, void* scratch, size_t scratch_bytes,
                            void* hip_stream);

/* Empties rows: every page they name loses a reference, their entries become
 * -1 and their lens 0.  info = {entries released, pages that became free}. */
ssba_status ssba_pages_release(const ssba_cache* c, const ssba_pages* p, int32_t n, const int32_t* row, int32_t* info,
                               void* scratch, size_t scratch_bytes, void* hip_stream);

/* Moves pages in use to the low end of the pool: with L pages in use, the k-th
 * page in use numbered L or more goes to the k-th free one below L, all layers.
 * table_out and refs_out receive the new table and counts (they may be table
 * and refs themselves).  info = {L, pages moved}. */
ssba_status ssba_pages_compact(const ssba_cache* c, const ssba_pages* p, int32_t* table_out, int32_t* refs_out,
                               int32_t* info, void* scratch, size_t scratch_bytes, void* hip_stream);

/* Copies pages of all layers, keys, values, scales and means:
 * to[dst[j]] = from[src[j]].  The caches differ in `pages` and arrays only; they
 * may be one.  Pairs outside the caches are passed over; a page must not be
 * named twice in dst, nor in src and dst of one cache. */
ssba_status ssba_pages_copy(const ssba_cache* from, const ssba_cache* to, int32_t n, const int32_t* src,
                            const int32_t* dst, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SSBA_CACHE_H_ */
