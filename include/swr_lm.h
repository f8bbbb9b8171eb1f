/*
 * swr_lm.h -- C ABI of the operators that a recurrent language model is made of
 * around the recurrence, its norms and projections, from its tokens to what it
 * learns from: the embedding of tokens and its gradient, the short causal
 * convolution and the selective state space scan of a mixer (for training, for
 * prompts and for single tokens), and the log probabilities of given tokens with
 * their gradient.  Part of the same library as swr.h, whose conventions hold here
 * too:
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
 * validation returns one of swr.h's negative SWR_ERR_* codes and touches
 * nothing.  Values that only the device holds (tokens, lengths) are checked by
 * the kernels: none of them can make one read or write out of bounds.
 *
 * Strides are in elements and may not be negative; elements of the innermost
 * dimension are contiguous.  Pointers are aligned to their elements (rows that
 * are 16-byte aligned are read fastest), workspaces to 16 bytes.  Sums and
 * states are in float32; each output is rounded once, as it is stored.  Sums have a fixed
 * order: repeated calls give the same bits.
 *
 * Overlaps.  Outputs share no element with an input or another output unless said
 * otherwise.  The convolution's y and dx, the scan's y and dlogits may lie between
 * the elements of inputs of the same strides, as parts of one tensor's rows; the address
 * ranges of all other outputs, and beside inputs of other strides, have to be apart.
 */
#ifndef SWR_LM_H
#define SWR_LM_H

#include <stdint.h>

#include "swr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Embedding
 *
 *     y[i] = scale table[tokens[i]]              (rows of `width` elements)
 *     dtable[v] = scale sum over i with tokens[i] = v of dy[i]
 *
 * A token outside 0 .. vocab - 1 (padding) has a row of zeros and no part in the
 * gradient.  The gradient's rows of tokens that do not occur are zeros.  A token's
 * rows of dy are added in their order, in pieces of at most 16 rows whose sums are then
 * added in four runs, the runs in order, in float32.
 * ------------------------------------------------------------------------ */

typedef struct swr_embed {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of table and y, or of dy: SWR_DTYPE_F32 or SWR_DTYPE_BF16 */
    int32_t out_dtype;         /* of dtable: dtype or SWR_DTYPE_F32 (forward: dtype)       */
    int32_t token_bytes;       /* of a token: 4 (int32) or 8 (int64)                       */
    int64_t tokens, vocab, width;
    int64_t st;                /* row stride of table, or of dtable                        */
    int64_t sy;                /* row stride of y, or of dy                                */
    float scale;               /* finite                                                  */
    int32_t reserved;          /* must be 0                                               */
} swr_embed_t;

int swr_embedding(const swr_embed_t* e, const void* tokens, const void* table, void* y, void* stream);

int swr_embedding_backward(const swr_embed_t* e, const void* tokens, const void* dy, void* dtable, void* workspace,
                           void* stream);

/* Bytes of workspace that the backward needs, or an SWR_ERR_* code. */
int64_t swr_embedding_workspace_bytes(const swr_embed_t* e);

/* ------------------------------------------------------------------------
 * Short causal convolution
 *
 * Of each channel of x [B, T, C] with its own `taps` weights (1 to 8), w [C, taps]:
 *
 *     pre[t, c] = bias[c] + sum_k w[c, k] x[t - taps + 1 + k, c]
 *     y = pre / (1 + exp(-pre))  with SWR_CONV_SILU, else pre
 *
 * x before the first token is the state [B, taps - 1, C] (oldest token first), or
 * zero without one.  With `lengths`, batch b has lengths[b] tokens (taken within 0 and T): y, and
 * dx, are zero past them, and x and dy are not read there.
 * ------------------------------------------------------------------------ */

#define SWR_CONV_SILU 1u

typedef struct swr_conv {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of x, w, bias, state, y, dy, dx: F32 or BF16             */
    uint32_t flags;            /* SWR_CONV_SILU or 0                                      */
    int32_t taps;
    int64_t B, T, C;
    int64_t sx_b, sx_t;        /* strides of x                                            */
    int64_t sy_b, sy_t;        /* ... of y (the backward's dy)                            */
    int64_t sd_b, sd_t;        /* ... of the backward's dx                                */
} swr_conv_t;

/* w, bias (or NULL: zeros), state and state_out are contiguous.  lengths: NULL, or int32 [B].
 * state_out: NULL, or the last taps - 1 tokens of each batch (of the state and x); it may be
 * `state` itself (updated in place). */
int swr_causal_conv(const swr_conv_t* p, const void* x, const void* w, const void* bias, const void* state,
                    const int32_t* lengths, void* y, void* state_out, void* stream);

/* Gradients without a state: dx, and float32 dw [C, taps] and dbias [C] (or NULL). */
int swr_causal_conv_backward(const swr_conv_t* p, const void* x, const void* w, const void* bias, const void* dy,
                             const int32_t* lengths, void* dx, float* dw, float* dbias, void* workspace,
                             void* stream);

/* Bytes of workspace that the backward needs, or an SWR_ERR_* code. */
int64_t swr_causal_conv_workspace_bytes(const swr_conv_t* p);

/* ------------------------------------------------------------------------
 * Selective state space scan
 *
 * Every channel c of x [B, T, D] has N states (1 to 64), with rates A [D, N] and a
 * step of its own at every token; channels share B and C [B, T, G, N] in G groups
 * of D / G in a row:
 *
 *     s[t, c]    = softplus(dt[t, c] + bias[c])      (dt + bias without SWR_SCAN_SOFTPLUS)
 *     h[t, c, n] = exp(s[t, c] A[c, n]) h[t - 1, c, n] + s[t, c] x[t, c] B[t, n]
 *     v[t, c]    = sum_n C[t, n] h[t, c, n] + skip[c] x[t, c]
 *     y[t, c]    = v[t, c] z[t, c] / (1 + exp(-z[t, c]))     (v without z)
 *
 * h before the first token is h0, or zero.  With `lengths`, batch b has lengths[b] tokens (taken
 * within 0 and T): y, and the gradients, are zero past them, the inputs are not read
 * there, and the final state is the last token's.
 *
 * A token's own decay exp(s A) is a float32, and past its range infinite (times a state of 0 it is NaN); the
 * product of many tokens' may be past it, only the states count.  Gradients of a channel whose state is infinite or
 * NaN are infinite or NaN where the state counts, which of the two is not said.
 *
 * Carriers are the states before every SWR_SCAN_BLOCK tokens, float32
 * [B, ceil(T / SWR_SCAN_BLOCK), D, N]: the forward saves them for the backward.
 * ------------------------------------------------------------------------ */

#define SWR_SCAN_SOFTPLUS 1u
#define SWR_SCAN_BLOCK 16

typedef struct swr_scan {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of x, dt, B, C, z, y and their gradients: F32 or BF16    */
    uint32_t flags;            /* SWR_SCAN_SOFTPLUS or 0                                  */
    int32_t N;                 /* states a channel                                        */
    int64_t B, T, D, G;        /* G divides D                                             */
    int64_t sx_b, sx_t;        /* strides of x                                            */
    int64_t sdt_b, sdt_t;      /* ... of dt                                               */
    int64_t sz_b, sz_t;        /* ... of z (of no account without z)                    */
    int64_t sy_b, sy_t;        /* ... of y (the backward's dy)                            */
    int64_t sB_b, sB_t, sB_g;  /* ... of B                                                */
    int64_t sC_b, sC_t, sC_g;  /* ... of C                                                */
} swr_scan_t;

/* The scan's inputs.  A, bias, skip (float32) and h0 (float32 [B, D, N]) are contiguous; bias,
 * skip, z, h0 and lengths (int32 [B]) may be NULL. */
typedef struct swr_scan_inputs {
    const void *x, *dt;
    const float* A;
    const void *B, *C;
    const float *bias, *skip;
    const void* z;
    const float* h0;
    const int32_t* lengths;
} swr_scan_inputs_t;

/* Forward.  carriers and h_last (float32 [B, D, N];
 * it may be h0 itself, updated in place) may be NULL. */
int swr_selective_scan(const swr_scan_t* p, const swr_scan_inputs_t* in, void* y, float* carriers, float* h_last,
                       void* workspace, void* stream);
int64_t swr_selective_scan_workspace_bytes(const swr_scan_t* p);

/* Gradients of every input, all contiguous: dx, ddt, dz [B, T, D] and dB, dC [B, T, G, N] of
 * p's dtype; dA [D, N], dskip, dbias [D] and dh0 [B, D, N] float32.  dz is there where z is, dskip where skip is, dbias
 * where bias is (NULL otherwise); dh0 may be NULL.  dh_last (float32 [B, D, N], or NULL) is the gradient of the
 * final state.  carriers are the forward's. */
typedef struct swr_scan_gradients {
    void *dx, *ddt;
    float* dA;
    void *dB, *dC;
    float *dbias, *dskip;
    void* dz;
    float* dh0;
} swr_scan_gradients_t;

int swr_selective_scan_backward(const swr_scan_t* p, const swr_scan_inputs_t* in, const void* dy,
                                const float* carriers, const float* dh_last, const swr_scan_gradients_t* out,
                                void* workspace, void* stream);
int64_t swr_selective_scan_backward_workspace_bytes(const swr_scan_t* p);

/* ------------------------------------------------------------------------
 * Log probabilities
 *
 * Of rows of logits [rows, vocab], with z = scale logits:
 *
 *     lse = log sum_v exp(z[v]),  logp = z[token] - lse,  entropy = lse - sum_v p[v] z[v],  p = exp(z - lse)
 *
 * and the `top` largest z with their tokens, the largest first, equal ones by the
 * lower token (NaN counts as larger than every number).  A token outside 0 .. vocab - 1 (not
 * scored) has logp = 0 and no gradient by it.  Logits of -infinity have p = 0 and no
 * part in the entropy.  A row of nothing else has lse = -infinity, logp =
 * -infinity, entropy = 0 and no gradient; a row that holds NaN or +infinity has NaN there.
 * Where scale times the largest logit leaves float32, lse is an infinity of its sign; logp, entropy and the
 * gradient go by distances from the largest logit, and are as defined.
 * ------------------------------------------------------------------------ */

#define SWR_TOP_MOST 64

typedef struct swr_logprob {
    int32_t abi_version;       /* must be SWR_ABI_VERSION                                 */
    int32_t dtype;             /* of the logits and their gradient: F32 or BF16            */
    int32_t token_bytes;       /* of a token: 4 (int32) or 8 (int64)                       */
    int32_t top;               /* alternatives: 0 to SWR_TOP_MOST, at most vocab           */
    int64_t rows, vocab;
    int64_t sl;                /* row stride of the logits                                */
    int64_t sd;                /* ... of their gradient                                   */
    float scale;               /* positive, finite, also times log2 e (1 / temperature)    */
    int32_t reserved;          /* must be 0                                               */
} swr_logprob_t;

/* logp, lse, entropy: float32 [rows].  top_logp (float32) and top_tokens (int64): [rows, top], not read
 * without alternatives. */
int swr_log_probs(const swr_logprob_t* p, const void* logits, const void* tokens, float* logp, float* lse,
                  float* entropy, float* top_logp, int64_t* top_tokens, void* workspace, void* stream);

/* Bytes of workspace that swr_log_probs needs (it may be NULL where they are 0), or an SWR_ERR_* code. */
int64_t swr_log_probs_workspace_bytes(const swr_logprob_t* p);

/* The logits' gradient, of the gradients of logp, lse and entropy (float32 [rows]; each may be NULL):
 *     dlogits[v] = scale (dlogp ([v = token] - p[v]) + dlse p[v] - dentropy p[v] (log p[v] + entropy))
 * lse and entropy are the forward's (of rows with |lse| > 256, where float32 holds too little of it, or none, the sum
 * is taken anew).  dlogits may be the logits themselves. */
int swr_log_probs_backward(const swr_logprob_t* p, const void* logits, const void* tokens, const float* lse,
                           const float* entropy, const float* dlogp, const float* dlse, const float* dentropy,
                           void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SWR_LM_H */
