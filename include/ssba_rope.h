/*
 * ssba_rope.h -- C ABI of the rotary positions with several axes for AMD
 * Instinct MI355X (gfx950), in the same library as ssba.h: queries and keys
 * turned by their tokens' (time, height, width, ...) positions, and gradients
 * turned back.
 *
 * A pair (a, b) of channels on axis x with frequency f (radians a position)
 * turns by phi = pos[token][x] * f:
 *   a' = a cos phi - b sin phi,   b' = b cos phi + a sin phi
 * and with `inverse` by -phi, which is also the gradient of the turn: the
 * gradients of a' and b' turned back are those of a and b.
 *
 * phi is formed and reduced in 64 bits, so far positions keep their angles
 * (error of about 2^-53 |phi|); the cosine and sine and the products are fp32
 * (each within 2^-23), the result is rounded once to the tensors' type.
 *
 * Ownership, streams and errors as in ssba.h: the caller owns every buffer,
 * calls are asynchronous on `hip_stream`, checks come before any launch, and
 * nothing is allocated or kept between calls.
 */
#ifndef SSBA_ROPE_H_
#define SSBA_ROPE_H_

#include "ssba.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which channels make a pair: (2 j, 2 j + 1), or (j, j + D/2). */
typedef enum ssba_rope_pairs { SSBA_ROPE_ADJACENT = 0, SSBA_ROPE_HALVES = 1 } ssba_rope_pairs;

typedef struct ssba_rope {
  int32_t head_dim;          /* 64 or 128                                        */
  int32_t pairs;             /* ssba_rope_pairs                                  */
  int32_t axes;              /* positions a token has: 1 .. 4                    */
  const int32_t* axis;       /* host [head_dim / 2]: axis of each pair; -1: the pair stays as it is */
  const double* freq;        /* host [head_dim / 2]: radians a position, at most 2^20 in size */
} ssba_rope;

/* A tensor [batch][heads][rows][D] and where its turned values go; y may be x
 * itself with the same strides, else the two must not overlap.  Element
 * strides, channels contiguous; all three 0: contiguous.  bf16: 16-byte
 * aligned, strides multiples of 8; fp32: 4-byte aligned.  A packed
 * [rows][heads][D] array is batch 1 with its strides. */
typedef struct ssba_rope_tensor {
  int32_t heads;             /* 1 .. 65536                                       */
  const void* x;
  void* y;
  int64_t x_stride_b, x_stride_h, x_stride_t;
  int64_t y_stride_b, y_stride_h, y_stride_t;
} ssba_rope_tensor;

/* Turns n tensors (1 or 2: queries, and keys of another number of heads) of
 * `batch` x `rows` tokens by their positions: pos int32 (device), the axes of
 * token (b, t) at pos + b * pos_stride_b + t * pos_stride_t (elements,
 * pos_stride_b 0: one set for all).  Batch or rows 0: nothing is done. */
ssba_status ssba_rope_rotate(const ssba_rope* r, int32_t dtype, int32_t inverse, int32_t batch, int32_t rows,
                             const int32_t* pos, int64_t pos_stride_b, int64_t pos_stride_t, int32_t n,
                             const ssba_rope_tensor* tensors, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SSBA_ROPE_H_ */
