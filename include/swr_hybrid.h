/*
 * swr_hybrid.h -- C ABI of the operators that stand around the recurrence in
 * a hybrid model (Sec. 6: Phalanx and attention layers in turn, each between a
 * root-mean-square norm and projections): the normed residual stream, the
 * projections of decoded tokens with 4-bit weights, and attention over a paged
 * key-value cache with the tables that describe it.  Part of the same library
 * as swr.h, whose conventions hold here too:
 *
 * Ownership.  Every pointer is device memory owned by the caller.  The library
 * allocates no memory and keeps no state; calls from several host threads are
 * safe.  Calls that need a workspace say how many bytes; it needs no
 * initialisation, its contents are scratch, and two calls in flight at once
 * need two.  Outputs are fully overwritten unless said otherwise.
 *
 * Asynchrony.  Work is enqueued on `stream` (a hipStream_t passed as void*;
 * NULL = the default stream) and the call returns without waiting.
 *
 * Errors.  Arguments are validated before any HIP runtime call; a failed
 * validation returns one of swr.h's negative SWR_ERR_* codes (an
 * SWR_ERR_BLOCK here is a page size out of range) and touches nothing.
 * Values that only the device holds (lengths, tables, slots) are checked by
 * the kernels: none of them can make one read or write out of bounds.
 *
 * Strides are in elements unless said otherwise and may not be negative;
 * `es` below is an element's size in bytes.
 */
#ifndef SWR_HYBRID_H
#define SWR_HYBRID_H

#include <stdint.h>

#include "swr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit floating point of 4 exponent and 3 mantissa bits, largest value 448,
 * no infinities (where a call says that it takes it). */
#define SWR_DTYPE_FP8 2

/* ------------------------------------------------------------------------
 * Residual addition and root-mean-square norm
 *
 * Rows of `width` elements, `outer` times `inner` of them (a [B, T, width]
 * tensor; outer = 1 for [rows, width]), elements of a row contiguous:
 *
 *     h = x + r                                     (h = x without r)
 *     y = h / sqrt(mean(h^2) + eps) * weight
 *
 * The sum, the mean and y are in float32 from the unrounded h; h and y are each
 * rounded once, as they are stored.  Every tensor has its own strides of the outer and
 * inner row index; no alignment beyond an element's is needed (16-byte aligned
 * rows are read fastest).
 * ------------------------------------------------------------------------ */

typedef struct swr_norm {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of x, r, h, dy, dh, dx: SWR_DTYPE_F32 or SWR_DTYPE_BF16  */
    int32_t weight_dtype;      /* of weight: the same, or SWR_DTYPE_F32                   */
    int32_t out_dtype;         /* of y: dtype, or SWR_DTYPE_FP8 with a scale per row       */
    int64_t outer, inner, width;
    float eps;                 /* not negative, finite                                    */
    int32_t reserved;          /* must be 0                                               */
    int64_t sx_o, sx_i;        /* row strides of x (the backward's h)                      */
    int64_t sr_o, sr_i;        /* ... of the residual (the backward's dh)                  */
    int64_t sh_o, sh_i;        /* ... of h (the backward's dx)                             */
    int64_t sy_o, sy_i;        /* ... of y (the backward's dy)                             */
} swr_norm_t;

/* Forward.  residual and h may be NULL (without a residual, h is a copy of x), and then
 * their strides are not read; so may the backward's dh.
 * With out_dtype SWR_DTYPE_FP8, y holds q and scale [outer * inner] float32
 * receives s, with  s = max|y| / 448  over the row and  q = y / s  rounded to
 * nearest even (a row of zeros has s = 0 and q = 0; a row that holds a NaN has
 * s = NaN); scale is not read otherwise.  h may be x or residual itself
 * (updated in place: same address and strides). */
int swr_rms_norm(const swr_norm_t* norm, const void* x, const void* residual, const void* weight, void* y,
                 float* scale, void* h, void* stream);

/* Backward at the stored h: with n = h / sqrt(mean(h^2) + eps) and g = dy * weight,
 *     dx = (g - n mean(g n)) / sqrt(mean(h^2) + eps) + dh
 *     dweight = sum over rows of dy n
 * where dh (or NULL) is the gradient that reaches h on its other ways; dx is the
 * gradient of x and of the residual alike.  dweight [width] is float32, summed in
 * a fixed order (repeated calls give the same bits).  out_dtype must be dtype.
 * dx may be dy or dh itself. */
int swr_rms_norm_backward(const swr_norm_t* norm, const void* h, const void* weight, const void* dy,
                          const void* dh, void* dx, float* dweight, void* workspace, void* stream);

/* Bytes of workspace that the backward needs (16-byte aligned), or an SWR_ERR_* code. */
int64_t swr_rms_norm_workspace_bytes(const swr_norm_t* norm);

/* ------------------------------------------------------------------------
 * Projections with 4-bit weights
 *
 *     y[m, n] = s[m] sum_k x[m, k] W[n, k],   W[n, k] = value(code[n, k]) 2^(power[n, k / 32] - 127)
 *
 * A code's low three bits stand for 0, 0.5, 1, 1.5, 2, 3, 4, 6 and its high bit
 * for the sign (4-bit floating point of 2 exponent bits and 1 mantissa bit);
 * groups of 32 weights of a row share a power of two, stored as its exponent
 * plus 127 (0 to 252; 255 makes the group NaN; 253 and 254 hold weights beyond
 * float32's range).  Two codes share a byte, the even k in its low half.  A row of codes has ceil(K / 32) groups of 16 bytes, codes past K are
 * not used, and starts 16-byte aligned.  Sums are in float32.  Meant for the
 * few rows of a decoding step (weights are read once for every 32 rows of x; for every 16 of
 * bf16 rows of 4097 to 8192 elements and of float32 rows of 1025 to 2048).
 * ------------------------------------------------------------------------ */

typedef struct swr_fp4 {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of x (of w in swr_fp4_pack): F32, BF16, or (x) FP8       */
    int32_t out_dtype;         /* of y: SWR_DTYPE_F32 or SWR_DTYPE_BF16                    */
    int32_t reserved;          /* must be 0                                               */
    int64_t M, N, K;           /* rows of x, rows of W, elements of both                   */
    int64_t sx;                /* row stride of x (of w); elements of a row are contiguous */
    int64_t sy;                /* row stride of y                                         */
    int64_t sc, sp;            /* row strides of codes and powers, in bytes                */
} swr_fp4_t;

/* y of x, codes and powers.  scale: NULL, or s [M] float32 (1 without it). */
int swr_fp4_linear(const swr_fp4_t* p, const void* x, const float* scale, const void* codes, const void* powers,
                   void* y, void* stream);

/* Codes and powers of w [N, K] (F32 or BF16; M, sy and out_dtype are not
 * read): each group's power is the least that leaves no weight above 6, within
 * 1 to 252, and each weight's code the nearest value (ties to the even code);
 * codes past K are zero.  A group that holds an infinity or a NaN has power 255. */
int swr_fp4_pack(const swr_fp4_t* p, const void* w, void* codes, void* powers, void* stream);

/* ------------------------------------------------------------------------
 * Paged key-value cache
 *
 * A layer's cache is `pages` pages of `page_size` tokens; request i's token at
 * position t lies on page table[i][t / page_size] at t % page_size.  A slot is
 * page * page_size + offset.  Pages are handed out from the top of a stack of
 * free page numbers.
 * ------------------------------------------------------------------------ */

typedef struct swr_tables {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t reserved;          /* must be 0                                               */
    int64_t batch;             /* requests                                                */
    int64_t max_pages;         /* columns of the table                                    */
    int64_t st;                /* the table's row stride                                  */
    int64_t page_size;         /* 1 to 65536                                              */
    int64_t tokens;            /* entries of slots                                        */
    int64_t free_pages;        /* entries of the free stack                               */
} swr_tables_t;

/* The step's tables from the requests' lengths: request i, of lengths[i] tokens
 * so far, gets new_tokens[i] more (numbers below 0 count as 0).  Pages within
 * max_pages that these start are taken in order of requests and positions, the first from
 * free_stack[*free_count - 1] (a count is taken within 0 and free_pages), and written to the table [batch, max_pages];
 * its other entries stay.  Outputs:
 *     starts [batch + 1]   new tokens before each request, and of all
 *     slots [tokens]       slot of each new token, request by request; entries
 *                          past the last new token are -1
 *     new_lengths [batch]  lengths[i] + new_tokens[i]
 *     new_free_count [1]   free pages left
 * A page that the stack no longer holds is -1 in the table, and a token on such a page, on a
 * page whose table entry is negative, or past max_pages has slot -1.  lengths,
 * new_tokens, free_stack, free_count, table, starts, new_lengths and new_free_count
 * are int32, slots is int64. */
int swr_block_tables(const swr_tables_t* p, const int32_t* lengths, const int32_t* new_tokens,
                     const int32_t* free_stack, const int32_t* free_count, int32_t* table, int64_t* slots,
                     int32_t* starts, int32_t* new_lengths, int32_t* new_free_count, void* stream);

/* A layer's cache, [pages, page_size, heads, D] with the channels contiguous and
 * the same strides for keys and values.  D: a multiple of 16 up to 256.  Every
 * pointer, and every stride of this struct and of the calls' other [.., D]
 * tensors, must be a multiple of 16 bytes; the last element lies within 2^36
 * bytes. */
typedef struct swr_cache {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of the cache, q, k, v and y: SWR_DTYPE_F32 or BF16       */
    int64_t pages, page_size;  /* page_size 1 to 65536                                    */
    int64_t heads, D;          /* key-value heads, channels                               */
    int64_t s_page, s_token, s_head;
} swr_cache_t;

/* New keys and values into their slots: k and v are [tokens, heads, D] with
 * strides sk[0..1] and sv[0..1] (token, head), slots int64 [tokens].  A token whose
 * slot is not within the cache is left out; the slots of one call are distinct.  The two
 * caches may be parts of one allocation, between each other's elements. */
int swr_cache_append(const swr_cache_t* cache, int64_t tokens, const int64_t* sk, const int64_t* sv, const void* k,
                     const void* v, const int64_t* slots, void* k_cache, void* v_cache, void* stream);

typedef struct swr_paged {
    swr_cache_t cache;
    int64_t batch;             /* requests, each with one query token                     */
    int64_t q_heads;           /* a multiple of cache.heads: q_heads / heads share a key head */
    int64_t max_pages, st;     /* columns and row stride of the table                     */
    int64_t window;            /* 0: all positions; else the last `window` of them         */
    int64_t sq_b, sq_h;        /* strides of q [batch, q_heads, D]                         */
    int64_t sy_b, sy_h;        /* strides of y                                            */
    float scale;               /* of the products q . k; finite, also times log2 e         */
    int32_t reserved;          /* must be 0                                               */
} swr_paged_t;

/* Attention of one query token a request over its cached tokens:
 *     y[i, h] = sum_t p_t V[t] / sum_t p_t,   p_t = exp(scale q[i, h] . K[t])
 * over positions max(0, lengths[i] - window) .. lengths[i] - 1 and key head
 * h / (q_heads / heads).  A position whose page is not within the cache, or past
 * max_pages, is left out; a request with no position left has y = 0 (one whose positions
 * all have a product of -infinity has 0 / 0).
 * lse: NULL, or float32 [batch, q_heads] (contiguous) that receives log(sum_t p_t)
 * (-infinity for no position).  lengths and table are int32.  Products, softmax and sums in float32;
 * results do not depend on other requests beyond float32 rounding order. */
int swr_paged_attention(const swr_paged_t* p, const void* q, const void* k_cache, const void* v_cache,
                        const int32_t* table, const int32_t* lengths, void* y, float* lse, void* workspace,
                        void* stream);

/* Bytes of workspace that swr_paged_attention needs (16-byte aligned; it may be
 * NULL where they are 0), or an SWR_ERR_* code. */
int64_t swr_paged_workspace_bytes(const swr_paged_t* p);

#ifdef __cplusplus
}
#endif
#endif /* SWR_HYBRID_H */
