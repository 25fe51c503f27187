/*
 * ii_ops.h -- running a model on the weights a load left in HBM: products
 * with its matrices, its key/value cache, attention over that cache.
 *
 * Conventions, beside those of ii.h:
 *   - Every pointer is device memory (or pinned host memory that the device
 *     sees at the same address); each range an operator touches is checked to
 *     lie inside one such allocation (II_EINVAL), and what it writes not to
 *     meet what it reads (II_EOVERLAP).
 *   - Strides are in elements, the last axis is contiguous. The strides of
 *     inputs may be zero (a broadcast); rows of outputs may not meet.
 *   - Work is enqueued on `stream` and the call returns; nothing waits and
 *     nothing allocates, so calls may be captured into a graph. The memory
 *     must stay allocated until `stream` passes the call.
 *   - `work` is scratch the caller owns, for results of work that is split
 *     over a long axis: 16-byte aligned, zero-filled once before its first
 *     use. A call leaves it fit for the next one on the same stream; calls
 *     that may overlap on different streams need scratch of their own. NULL
 *     (0 bytes) means that nothing is split, which is slower for few rows.
 *     II_WORK_BYTES is as much as any call makes use of; that much of it may
 *     not meet what else the call reads or writes (II_EOVERLAP). The same inputs,
 *     strides and work_bytes give the same bits.
 */
#ifndef II_OPS_H
#define II_OPS_H

#include "ii.h"

#ifdef __cplusplus
extern "C" {
#endif

#define II_WORK_BYTES (64u << 20)

/* ---- activations ------------------------------------------------------- */
enum {
    II_ACT_NONE = 0,
    II_ACT_RELU = 1, /* max(y, 0) */
    II_ACT_SILU = 2, /* y / (1 + exp(-y)) */
    II_ACT_GELU = 3  /* y (1 + erf(y / sqrt(2))) / 2 */
};

/*
 * ii_linear -- a product with a weight matrix as a checkpoint stores it
 * ([n, k], row-major), and what follows it in a decoder layer:
 *
 *   y[i][j]   = sum_k x[i][k] w[j][k] + bias[j]
 *   z[i][j]   = sum_k x[i][k] w2[j][k] + bias2[j]        (if w2)
 *   out[i][j] = act(y[i][j]) * z[i][j] + residual[i][j]
 *
 * Products, sums and the epilogue are held in 32 bits; out is rounded once.
 *
 *   dtype      of x, w, w2, bias, bias2, residual: II_BF16 or II_F16.
 *   out_dtype  dtype or II_F32.
 *   m, n, k    any sizes from 0 to 2^31 - 1; with k = 0 the sums are 0.
 *   w2         NULL: no gate (bias2 must be NULL too).
 *   bias, bias2, residual   NULL: none. residual may be out itself.
 * Rows whose address and stride are multiples of 16 bytes, with k a multiple
 * of 8, go into matrix instructions or LDS as they are read; others through
 * registers first, which takes 1.5 to 2.2 times as long.
 * Errors: II_EINVAL, II_EALIGN (an address not a multiple of its element),
 * II_EOVERFLOW, II_EOVERLAP, II_EHIP.
 */
typedef struct ii_linear_args {
    int32_t dtype, out_dtype, act, reserved; /* reserved: 0 */
    int64_t m, n, k;
    const void* x;
    int64_t x_stride;
    const void* w;
    int64_t w_stride;
    const void* w2;
    int64_t w2_stride;
    const void* bias;
    const void* bias2;
    const void* residual;
    int64_t residual_stride;
    void* out;
    int64_t out_stride;
    void* work;
    uint64_t work_bytes;
} ii_linear_args;

int ii_linear(const ii_linear_args* args, hipStream_t stream);

/*
 * A paged key/value cache: `pages` pages of `page` tokens, each token `heads`
 * heads of `dim` elements for keys and as many for values. The element of
 * page p, head h, token t, position d lies at
 * p * page_stride + h * head_stride + t * token_stride + d.
 *
 * With dtype II_FP8_E4M3 every 32 consecutive elements of a head share a
 * scale 2^(s - 127), s (1 to 254) the byte at p * scale_page_stride +
 * h * scale_head_stride + t * scale_token_stride + d / 32 of k_scale or
 * v_scale; an element's value is its code times that scale. Memory of zeros
 * holds zeros. Scales that are powers of two cost an 8-bit float no precision,
 * and make every kept value exact in bf16, but one: magnitudes above
 * 248 * 2^120 (3.3e38) are kept as 2^128, which bf16 has as infinity.
 *
 *   dtype   II_BF16, II_F16 (as the activations) or II_FP8_E4M3.
 *   dim     64 or 128.
 *   page    a power of two.
 * Addresses and strides are multiples of 16 bytes (of dim / 32 bytes for the
 * scales).
 */
typedef struct ii_cache {
    int32_t dtype, heads, dim, page;
    int64_t pages;
    void* k;
    void* v;
    uint8_t* k_scale; /* NULL unless dtype is II_FP8_E4M3 */
    uint8_t* v_scale;
    int64_t page_stride, head_stride, token_stride;
    int64_t scale_page_stride, scale_head_stride, scale_token_stride;
} ii_cache;

/*
 * Keys and values of `tokens` tokens in the activations' type, and the slots
 * they have in a cache: slot s is token s mod page of page s / page.
 * Addresses and strides of k and v are multiples of 16 bytes.
 */
typedef struct ii_tokens {
    int32_t dtype, reserved; /* II_BF16 or II_F16; 0 */
    int64_t tokens;
    void* k;
    int64_t k_token_stride, k_head_stride;
    void* v;
    int64_t v_token_stride, v_head_stride;
    const int64_t* slots;
} ii_tokens;

/*
 * ii_cache_write -- put tokens into a cache, quantising them if it is
 * II_FP8_E4M3: the scale of 32 elements is the least power of two 2^e, e from
 * -126 to 120, with |x| <= 448 * 2^e for every finite x among them, the codes
 * x / 2^e rounded to nearest, ties to even. NaN and infinities become NaN and
 * leave the scale alone. For II_F16 tokens no value above 61440 is kept (the
 * next, 65536, does not fit the type).
 * Tokens whose slot is negative or past the last page are left out. Two
 * tokens of one call must not have the same slot. The cache's arrays may lie in
 * one buffer in any order of axes, but not meet (II_EOVERLAP).
 */
int ii_cache_write(const ii_cache* cache, const ii_tokens* from, hipStream_t stream);

/*
 * ii_cache_read -- take tokens out of a cache into `to` (its k and v are
 * written): codes times scales, exact (values under the type's least normal
 * are rounded to it). Slots that are negative or past the last page give zeros.
 */
int ii_cache_read(const ii_cache* cache, const ii_tokens* to, hipStream_t stream);

/*
 * ii_attend -- attention of a ragged batch of new tokens over a paged cache
 * that already holds their keys and values.
 *
 * Sequence b's queries are rows [q_start[b], q_start[b + 1]) of q (row b
 * alone if q_start is NULL); they are its last tokens: with length_b =
 * lengths[b] keys, query i of n sits at position p = length_b - n + i and sees
 * the keys j with p - window < j <= p (all j <= p if window is 0). Key j lies
 * in token j mod page of page pages[b * pages_stride + j / page]. Query head h
 * uses cache head h / (heads / cache->heads).
 *
 *   out = sum_j softmax_j(scale q . k_j) v_j;   zero where no key is seen.
 *
 * Scores, softmax statistics and sums are held in 32 bits; the weights are
 * rounded to the activations' type for the product with the values, where f16
 * keeps 11 bits of those down to 2^-27 of a row's largest.
 *
 *   dtype     of q and out: II_BF16 or II_F16; the cache's, unless that is
 *             II_FP8_E4M3.
 *   heads     query heads, a multiple of cache->heads.
 *   rows      rows of q and out, rows * heads at most 2^30. q_start is read on
 *             the device; rows it puts outside [0, rows) are left out.
 *   seqs      sequences; lengths has as many, q_start one more.
 *   columns   columns of the page table. Keys past columns * page, and keys
 *             of pages that are negative or not below cache->pages, are not
 *             seen.
 *   max_q     the most queries of a sequence, max_len the most keys (0:
 *             columns * page). They only shape the launch: more of either
 *             costs time, not correctness.
 *   scale     of the scores, any finite float.
 */
typedef struct ii_attend_args {
    int32_t dtype, heads;
    int64_t rows, seqs;
    const void* q;
    int64_t q_row_stride, q_head_stride;
    void* out;
    int64_t out_row_stride, out_head_stride;
    const int32_t* pages;
    int64_t pages_stride, columns;
    const int32_t* lengths;
    const int32_t* q_start;
    int64_t max_q, max_len, window;
    float scale;
    int32_t reserved; /* 0 */
    void* work;
    uint64_t work_bytes;
} ii_attend_args;

int ii_attend(const ii_attend_args* args, const ii_cache* cache, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif
