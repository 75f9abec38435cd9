/*
 * tas_fp4.h - C ABI of a serving iteration in four bits on MI355X: the KV cache
 * of tas_step.h held in four bits, and products with weights held so.
 *
 * FOUR BITS. 32 adjacent elements of a row are a block with one scale, 2^e, held
 * as the byte e + 127 (255: every element of the block is NaN). An element is a
 * sign bit and three bits that stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6, times the
 * scale; elements 2j and 2j + 1 are the low and the high half of byte j of the
 * row's codes. This is the chip's own format: it converts two elements an
 * instruction, exactly.
 *
 * ROUNDING to it: e is the smallest exponent with max |x| < 7 * 2^e over the
 * block (from 7 on the largest would round to 8, which there is not; on normal
 * values the mean square error is 1.25 % so, 1.32 % with the largest power of two
 * below, 1.33 % with the smallest that holds it), but from -125 to 125 for
 * bfloat16 and -23 to 13 for float16: there every value that a block can stand
 * for is one of the 16-bit type. An element goes to the nearest of the eight
 * magnitudes, from the middle of two to the even code, beyond the largest to the
 * largest. A block with a value that is infinite or NaN has the scale 255 and
 * codes of 0.
 *
 * READING it in a 16-bit type: a scale beyond those exponents (from elsewhere)
 * gives values that are rounded as that type rounds, or infinite.
 *
 * Conventions as in tas_step.h: negative return codes, no exceptions, tensors are
 * caller-owned device memory, everything is enqueued on the caller's stream (any
 * stream, capturable) and allocates nothing.
 */
#ifndef TAS_FP4_H
#define TAS_FP4_H

#include <stddef.h>
#include <stdint.h>

#include "tas_step.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of adjacent bytes: row (i0, i1, i2) lies at p + i0 * stride[0] +
 * i1 * stride[1] + i2 * stride[2] (bytes). */
typedef struct tas_rows {
    void *p;
    int64_t stride[3];
} tas_rows;

/* One layer's cache; rows (block, head, token of the block): head_dim / 2 bytes of
 * codes, head_dim / 32 of scales. Codes 16-byte aligned, strides multiples of 16;
 * scales aligned to their row, strides multiples of it. Strides of a block or head
 * below 2^31, of a token at most 2^24. For tas_fp4_append no two bytes of the pool
 * may lie in one place, as for tas_step_append. */
typedef struct tas_cache_fp4 {
    tas_rows k, v, k_scale, v_scale;
} tas_cache_fp4;

/* As tas_append, with a cache in four bits. */
typedef struct tas_append_fp4 {
    int32_t dtype, rot_dim, interleaved;
    float eps;
    const void *qkv;
    int64_t qkv_stride;
    void *q_out;
    int64_t q_out_stride;
    const void *q_weight, *k_weight;
    const float *cos, *sin;
    int64_t positions;
    tas_cache_fp4 cache;
} tas_append_fp4;

/* As tas_attention, with a cache in four bits. */
typedef struct tas_attention_fp4 {
    int32_t dtype;
    float scale;
    const void *q;
    int64_t q_stride;
    void *out;
    int64_t out_stride;
    float *lse;
    tas_cache_fp4 cache;
} tas_attention_fp4;

/* Norm, rotate and append as tas_step_append: queries go to q_out, in 32 bits and
 * rounded once; keys and values are rounded to four bits, keys to the codes that
 * the formula has in 64 bits (so that the order of their norm's sum does not
 * decide between two), and go to the token's slots. TAS_EINVAL: as there, or the
 * cos, sin or weights overlap an output. */
int tas_fp4_append(tas_step *step, const tas_append_fp4 *a, void *stream);

/* Attention as tas_step_attention over the values that the cache stands for. (A
 * block that is NaN is a value that is not finite.) TAS_EINVAL: as there, or lse
 * overlaps another tensor. */
int tas_fp4_attention(tas_step *step, const tas_attention_fp4 *a, void *stream);

/* A tensor of n[0] * n[1] * n[2] rows of `cols` elements, cols a multiple of 32:
 * `x` in a 16-bit type (16-byte aligned, strides multiples of 16), `codes` and
 * `scales` (codes 4-byte aligned, strides multiples of 4); the stride of a dimension of one
 * says nothing. At most 2^35 - 2^11 elements. */
typedef struct tas_tensor_fp4 {
    int32_t dtype;                 /* of x: TAS_F16 or TAS_BF16                              */
    int32_t reserved;              /* 0                                                      */
    int64_t n[3], cols;
    tas_rows x, codes, scales;
} tas_tensor_fp4;

/* codes, scales <- x rounded to four bits. TAS_EINVAL: sizes or alignments out of
 * range, outputs whose rows overlap one another or x; TAS_EHIP. */
int tas_fp4_pack(const tas_tensor_fp4 *a, void *stream);
/* x <- the values that codes and scales stand for. Errors as tas_fp4_pack. */
int tas_fp4_values(const tas_tensor_fp4 *a, void *stream);

/* The values of a whole cache: k and v, [n_blocks][kv_heads][block_tokens][head_dim] in
 * a 16-bit type, 16-byte aligned, <- what the cache stands for, in one launch. */
typedef struct tas_cache_values_fp4 {
    int32_t dtype;                 /* of k and v                                             */
    int32_t head_dim;              /* 64 or 128                                              */
    int64_t n_blocks, kv_heads, block_tokens;
    tas_cache_fp4 cache;
    void *k, *v;
} tas_cache_values_fp4;
/* Errors as tas_fp4_values. */
int tas_fp4_cache_values(const tas_cache_values_fp4 *a, void *stream);

/* WEIGHTS: a matrix [rows][cols] in four bits, laid out once for the products, in
 * tas_fp4_weights_bytes bytes of device memory (0: sizes out of range: rows 1 ..
 * 2^24, cols a multiple of 32 up to 2^20). */
size_t tas_fp4_weights_bytes(int64_t rows, int64_t cols);
/* d_weights (256-byte aligned) <- the matrix of row-major codes (16-byte aligned,
 * stride in bytes a multiple of 16) and scales. */
int tas_fp4_weights(int64_t rows, int64_t cols, const void *codes, int64_t codes_stride,
                    const void *scales, int64_t scales_stride, void *d_weights, void *stream);

/* Arguments of tas_fp4_linear: y = x W^T, y[t][n] = sum over k of x[t][k] W[n][k]. */
typedef struct tas_linear_fp4 {
    int32_t dtype;                 /* of x and y                                             */
    int32_t reserved;              /* 0                                                      */
    int64_t tokens, rows, cols;    /* tokens 0 .. 2^24                                       */
    const void *x;                 /* [tokens][cols], 16-byte aligned                        */
    int64_t x_stride;              /* elements, a multiple of 8, at most 2^24                */
    const void *weights;           /* as tas_fp4_weights laid them out                       */
    void *y;                       /* [tokens][rows], 2-byte aligned                         */
    int64_t y_stride;              /* elements, below 2^31                                   */
} tas_linear_fp4;

/* The products of x's and W's values (W's are exact in 16 bits) are summed in 32
 * bits in an order that depends on the sizes alone, and rounded once. TAS_EINVAL:
 * an argument out of range or unaligned, y over x or the weights, more than 2^33 elements
 * of y (about: 2^21 tiles of 64 by 64). */
int tas_fp4_linear(const tas_linear_fp4 *a, void *stream);
/* Which of its kernels tas_fp4_linear takes for these sizes (0 on; tokens at least 1): for
 * tests and timings that have to reach each. Host only. TAS_EINVAL: sizes out of range. */
int tas_fp4_linear_kernel(int64_t tokens, int64_t rows, int64_t cols);
enum { TAS_FP4_LINEAR_KERNELS = 14 };

#ifdef __cplusplus
}
#endif
#endif
