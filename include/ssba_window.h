/*
 * ssba_window.h -- C ABI of causal attention with a sliding window and first
 * tokens that stay visible (sinks), forward and backward, for AMD Instinct
 * MI355X (gfx950), in the same library as ssba.h.  ssba_cache.h has the form
 * that reads a cache.
 *
 * Token i of a sequence sees the tokens j <= i with j < sinks or j > i -
 * window; it always sees itself.  With the group G = heads / kv_heads, query
 * heads h * G .. h * G + G-1 read kv head h:
 *   s_ij = scale q_i k_j,  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i)
 *   o_i = sum_j p_ij v_j
 *   delta_i = do_i o_i,  ds_ij = p_ij (do_i v_j - delta_i)
 *   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
 * where dk and dv also sum over the group's query heads, always in the same
 * order: results do not depend on atomics or on the order of workgroups.
 *
 * Sequences: a batch of equal ones, [batch][heads][seq][D] with any strides
 * (channels contiguous); or, with `cu`, packed ones: batch is 1, rows cu[s] ..
 * cu[s+1]-1 of the `seq` rows are sequence s (device int32 [seqs + 1], not
 * decreasing; read on the device, so a captured call replays with new lengths,
 * and whatever they hold, no access leaves the arrays).  Rows of no sequence
 * are neither read nor written.
 *
 * What a token does not see has no influence on its result, whatever it holds
 * (NaN and infinities too); the same holds for gradients.
 *
 * bf16: products of bf16 values with fp32 sums; probabilities and ds enter the
 * second products rounded to bf16 (half a step each, like the results; the ds of
 * dq as two bf16 terms where window + sinks is at most 1024).  fp32: values as
 * three bf16 terms, products within 2^-22 of exact ones, fp32 sums; of values
 * below 2^-110 the last bits are lost.  Softmax statistics are fp32: p of the
 * backward comes from lse, so it is off by about |lse| 2^-23, which scores of some
 * thousands begin to show.  Where a row's |lse| is 2^20 or more p is kept at most
 * 1, so that finite inputs have finite gradients, but says little else.  How the
 * work is split goes by the sizes of the call and max_len, and the rounding of
 * partial sums with it.
 *
 * Ownership, streams and errors as in ssba.h: the caller owns every buffer,
 * calls are asynchronous on `hip_stream`, checks come before any launch, and
 * nothing is allocated or kept between calls.  Calls that overlap in time must
 * not share a scratch buffer.
 */
#ifndef SSBA_WINDOW_H_
#define SSBA_WINDOW_H_

#include "ssba.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element strides of a [batch][heads][seq][D] array; all 0: contiguous.  bf16:
 * 16-byte aligned, strides multiples of 8; fp32: the same with multiples of 4. */
typedef struct ssba_strides {
  int64_t b, h, t;           /* t at most 2^20                                   */
} ssba_strides;

typedef struct ssba_window {
  int32_t batch;             /* sequences of equal length; packed: 1             */
  int32_t seq;               /* rows of each; packed: of all                     */
  int32_t heads, kv_heads;   /* heads a multiple of kv_heads; at most 65536      */
  int32_t head_dim;          /* 64 or 128                                        */
  int32_t dtype;             /* ssba_dtype of every tensor                       */
  int32_t window, sinks;     /* window >= 1, sinks >= 0                          */
  int32_t seqs;              /* packed: sequences, 1 .. 65535; else 0            */
  int32_t max_len;           /* packed: about the longest sequence (how work is split goes by it); 0: seq */
  float softmax_scale;       /* <= 0 selects 1 / sqrt(head_dim); at most 2^127   */
  const int32_t* cu;         /* packed: device int32 [seqs + 1]; else NULL       */
  ssba_strides q, k, v, o;   /* k, v: of kv_heads heads                          */
} ssba_window;

/* o and lse (fp32 [batch][heads][seq], contiguous; natural logarithm; NULL: not
 * wanted).  o must not overlap the inputs. */
ssba_status ssba_window_forward(const ssba_window* w, const void* q, const void* k, const void* v, void* o, float* lse,
                                void* hip_stream);

/* Strides of the backward's arrays: do_ that of dO, dq, dk, dv of the gradients. */
typedef struct ssba_window_grads {
  ssba_strides do_, dq, dk, dv;
} ssba_window_grads;

/* Device bytes of the scratch of ssba_window_backward. */
ssba_status ssba_window_backward_workspace_size(const ssba_window* w, size_t* scratch_bytes);

/* Gradients of q, k and v from that of o, with the forward's o and lse.  The
 * gradients must not overlap each other or the inputs; `scratch` 16-byte aligned. */
ssba_status ssba_window_backward(const ssba_window* w, const ssba_window_grads* g, const void* q, const void* k,
                                 const void* v, const void* o, const void* dout, const float* lse, void* dq, void* dk,
                                 void* dv, void* scratch, size_t scratch_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SSBA_WINDOW_H_ */
