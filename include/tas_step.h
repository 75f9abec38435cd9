/*
 * tas_step.h - C ABI of the attention part of one serving iteration on MI355X.
 *
 * The simulator of tas.h prices ExecuteOneStep (arXiv 2606.18431, Algorithm 1:
 * "run the prefill chunks and decode steps; update KV and token counters") by
 * an integer cost model. These entry points do what that price stands for to
 * the batch a scheduler formed: the new tokens' keys and values go to the paged
 * KV cache whose blocks the simulator counts, and every new token attends to
 * its request's context there.
 *
 * A BATCH is n_req requests. Request i brings n_new[i] new tokens (1: a decode
 * step; more: a prefill chunk) and has kv_len[i] tokens of context of its own,
 * the new ones included, in the blocks blocks[i][0], blocks[i][1], ... Token y
 * of the context lies in blocks[i][y / block_tokens] at y % block_tokens. Runs
 * of adjacent requests may share a PREFIX (the simulator's prefix-cache hits):
 * group g is the requests prefix_first[g] .. prefix_first[g + 1] - 1, and its
 * prefix_len[g] tokens precede the own context of each of them. The batch's T
 * new tokens are numbered request by request; token j of request i has position
 *     prefix_len[g] + kv_len[i] - n_new[i] + j.
 *
 * A STEP context is the plan of one batch: made by tas_step_create when the
 * scheduler has formed the batch, bound to device memory by tas_step_bind (or
 * tas_step_attach), used for every layer of the model.
 *
 * Conventions as in tas.h: negative return codes (TAS_E*), no exceptions;
 * batch arrays are host memory, read only during the call; d_* and the tensor
 * pointers are caller-owned device memory; tas_step_append and
 * tas_step_attention only enqueue kernels on the caller's stream (any stream,
 * capturable) and allocate nothing. One step's attention calls share its
 * workspace: enqueue them on one stream, or order them.
 */
#ifndef TAS_STEP_H
#define TAS_STEP_H

#include <stddef.h>
#include <stdint.h>

#include "tas.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TAS_F16 = 0, TAS_BF16 = 1 };

typedef struct tas_batch {
    int32_t heads, kv_heads;       /* heads a multiple of kv_heads, >= 1; heads <= 1024      */
    int32_t head_dim;              /* 64 or 128                                              */
    int32_t block_tokens;          /* a power of two, 16 .. 4096                             */
    int32_t n_req, n_blocks;       /* requests >= 1; blocks in the pool >= 1                 */
    int32_t causal;                /* 1: a token sees its context up to itself; 0: all of it */
    int32_t n_prefix;              /* groups, 0: no prefixes                                 */
    const int32_t *n_new;          /* HOST [n_req] >= 0                                      */
    const int32_t *kv_len;         /* HOST [n_req] >= 0                                      */
    const int32_t *blocks;         /* HOST [n_req][blocks_stride]: only the entries that     */
    int64_t blocks_stride;         /*      kv_len reaches are read, each in [0, n_blocks)    */
    const int32_t *prefix_first;   /* HOST [n_prefix + 1], 0 = first <= ... <= last = n_req  */
    const int32_t *prefix_len;     /* HOST [n_prefix] >= 0                                   */
    const int32_t *prefix_blocks;  /* HOST [n_prefix][prefix_stride], as blocks              */
    int64_t prefix_stride;
} tas_batch;

/* One layer's cache: element (block, head, token of the block, d) of K lies at
 * k + block * k_block + head * k_head + token * k_token + d (elements); V
 * likewise. Pointers 16-byte aligned, strides multiples of 8, below 2^31, of a
 * token at most 2^24. For tas_step_append no two elements of the pool's K and V may
 * lie in one place: in the order of the strides, each is at least as long as what the
 * shorter ones span, and K and V have no element in common (they may alternate, by
 * blocks, heads, tokens or halves of a row). */
typedef struct tas_cache {
    void *k, *v;
    int64_t k_block, k_head, k_token;
    int64_t v_block, v_head, v_token;
} tas_cache;

/* Arguments of tas_step_append. Tensors of `dtype` unless said otherwise,
 * 16-byte aligned, token strides (elements) multiples of 8, heads of a token
 * adjacent: head h of token t at t * stride + h * head_dim. */
typedef struct tas_append {
    int32_t dtype;                 /* TAS_F16 or TAS_BF16                                    */
    int32_t rot_dim;               /* rotated elements of a head: 0, or a multiple of 16 up  */
                                   /* to head_dim                                            */
    int32_t interleaved;           /* pairs (2m, 2m + 1) instead of (m, m + rot_dim / 2)     */
    float eps;                     /* of the norm, >= 0                                      */
    const void *qkv;               /* [T][heads + 2 kv_heads][head_dim]: queries, keys, values */
    int64_t qkv_stride;
    void *q_out;                   /* [T][heads][head_dim]; may be qkv, with its stride      */
    int64_t q_out_stride;
    const void *q_weight, *k_weight; /* [head_dim] norm weights; both, or both NULL: no norm */
    const float *cos, *sin;        /* float [positions][rot_dim / 2], rows adjacent          */
    int64_t positions;             /* more than every new token's position                   */
    tas_cache cache;
} tas_append;

/* Arguments of tas_step_attention. */
typedef struct tas_attention {
    int32_t dtype;
    float scale;                   /* of the scores, positive; scale * log2(e) finite        */
    const void *q;                 /* [T][heads][head_dim]                                   */
    int64_t q_stride;
    void *out;                     /* [T][heads][head_dim]; may be q, with its stride        */
    int64_t out_stride;
    float *lse;                    /* float [T][heads]: log of the sum of exp(scores), or NULL */
    tas_cache cache;
} tas_attention;

typedef struct tas_step tas_step;

/* Validate and plan a batch (host only). TAS_EINVAL: a field out of range, a
 * block number outside the pool, more than 2^24 tokens or work for as many
 * workgroups, in a causal batch a block that new tokens of two requests, or two
 * pages of one, would be written to (without causality such a batch can be
 * attended, not appended); TAS_ENOMEM: no host memory. */
int tas_step_create(const tas_batch *batch, tas_step **out);
/* Bytes of device workspace that the step needs (plan and partial results). */
size_t tas_step_bytes(const tas_step *step);
/* Copy the plan to d_ws (256-byte aligned, at least tas_step_bytes) on the
 * stream, and wait for that: for all that the stream was given before, too. d_ws
 * must outlive the step's last call and stay untouched by others. TAS_EINVAL,
 * TAS_ENOMEM (ws_bytes too small), TAS_EHIP. */
int tas_step_bind(tas_step *step, void *d_ws, size_t ws_bytes, void *stream);
/* As tas_step_bind, for a caller that copies the plan itself and does not wait: host
 * only. What tas_step_plan gives has to lie at d_ws before the step's first call runs
 * (enqueued before it on its stream, or waited for). */
int tas_step_attach(tas_step *step, void *d_ws, size_t ws_bytes);
void tas_step_destroy(tas_step *step);
/* New tokens of the batch (T). */
int64_t tas_step_tokens(const tas_step *step);

/* Norm, rotate and append. For every new token, of its query and key heads u:
 *     u <- u / sqrt(mean(u^2) + eps) * weight       (with weights)
 *     (a, b) <- (a cos - b sin, b cos + a sin)      (each rotated pair)
 * queries go to q_out, keys and the unchanged values to the token's slot of the
 * cache. In 32 bits, rounded once. TAS_EINVAL: an argument out of range or
 * unaligned, a cache whose slots overlap, tensors that overlap, a batch with
 * kv_len[i] < n_new[i] or new tokens in one block, positions too small;
 * TAS_ESTATE: not bound (also below). */
int tas_step_append(tas_step *step, const tas_append *a, void *stream);

/* out = softmax(scale * q K^T) V of every new token and head, over the group's
 * prefix and the keys y < kv_len[i] of its own context (causal: y <= kv_len[i] -
 * n_new[i] + j); query head h reads key head h / (heads / kv_heads). Scores, maxima
 * and sums are held in 32 bits; the softmax's weights are rounded to the tensors'
 * type for the product with V, and the result once. A row without keys gives 0 and
 * lse -inf. What a row does not see does not reach it, whatever the slots hold; a
 * value that it sees and that is not finite makes its element not finite, or the
 * whole row NaN. TAS_EINVAL: an argument out of range or
 * unaligned, out over a part of q or of the cache. */
int tas_step_attention(tas_step *step, const tas_attention *a, void *stream);

/* The plan that tas_step_bind copies to the device: writes it to
 * host memory `buf` and its size to *bytes (with buf NULL, the size only). Host
 * only. TAS_EINVAL, TAS_ENOMEM (buf_bytes too small). */
int tas_step_plan(const tas_step *step, void *buf, size_t buf_bytes, size_t *bytes);

#ifdef __cplusplus
}
#endif
#endif
