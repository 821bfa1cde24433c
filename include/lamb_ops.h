/*
 * lamb_ops.h -- C ABI of the operators around the optimizer step, for AMD
 * Instinct MI355X (gfx950): Newton-Schulz orthogonalization and the Muon step
 * for a model's matrices, softmax cross entropy against a vocabulary table with
 * its gradients, and a token table's lookup with its gradient. Same library,
 * status codes and conventions as lamb_mi355x.h: pointers are device pointers
 * unless marked host; the caller owns every tensor; arguments are validated on
 * the host before any HIP call; work is enqueued on `stream` and nothing is
 * synchronised, allocated or copied to the host (plan creation and destruction
 * aside); lamb_last_error() describes a failure. Nothing throws. Memory that a call
 * writes may not overlap any other of its operands (LAMB_EOVERLAP); operands of one row
 * stride may lie between each other's rows, as the column slices of a buffer do.
 */
#ifndef LAMB_OPS_H
#define LAMB_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "lamb_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of an operator's tensors. */
typedef enum lamb_dtype {
    LAMB_DTYPE_F32 = 0,
    LAMB_DTYPE_BF16 = 1, /* raw 16-bit patterns */
    LAMB_DTYPE_I32 = 2,  /* token ids */
    LAMB_DTYPE_I64 = 3   /* token ids */
} lamb_dtype;

/*
 * How the products of the Newton-Schulz iteration round their operands.
 *  LAMB_NS_SPLIT  to the sum of two 16-bit floats (22 bits), three products for one:
 *                 errors as of fp32 arithmetic that rounds a sum once in 32 terms.
 *  LAMB_NS_HALF   to one (11 bits). X, of norm 1, is so rounded to 2^-11 of itself at
 *                 most, and the iteration multiplies what is small in it by up to
 *                 |a|^steps (485 by default): the result is off by up to 0.3, beside
 *                 its own norm of about sqrt(min(rows, cols)) where most singular
 *                 values reach 1. Relative, as 2-norms: 1.3e-3 for independent entries,
 *                 4e-3 to 1.5e-2 for singular values that fall evenly over 2 to 6
 *                 decades, 4e-2 for rank 16 and noise of 2e-3 of it, 1.5e-1 where one
 *                 singular value outweighs all others together by a thousand. (The
 *                 rounding of a bf16 result is 1.7e-3.)
 */
typedef enum lamb_ns_precision { LAMB_NS_HALF = 0, LAMB_NS_SPLIT = 1 } lamb_ns_precision;

/*
 * The iteration: X = G / (||G||_F + eps), then `steps` times
 *   A = X X^T (or X^T X, on the shorter side),  X <- (a I + b A + c A A) X.
 * steps 1 to 64, eps >= 0 (with eps = 0 a matrix of zeros gives NaN), and a, b, c such
 * that no singular value that starts in [0, 1] passes 2.75, nor the polynomial
 * 7.75, on the way (LAMB_EINVAL): the iteration's 16-bit numbers hold no more.
 */
typedef struct lamb_ns_params {
    int32_t steps;
    float a, b, c;
    float eps;
    int32_t reserved; /* must be 0 */
} lamb_ns_params;

/* 5 steps of (3.4445, -4.7750, 2.0315), eps 1e-7. */
LAMB_API lamb_status lamb_ns_params_init(lamb_ns_params *params);

/*
 * One matrix to orthogonalize, row-major with rows `*_stride` elements apart
 * (>= cols, at most 2^36). rows and cols 1 to 2^20, aligned to their element. A row or column
 * vector is a matrix of short side 1. No output may share memory with an input of the plan
 * or another output, but for an input that has the output's address, type and
 * stride (in place).
 */
typedef struct lamb_matrix {
    const void *in;
    void *out;
    int64_t rows, cols;
    int64_t in_stride, out_stride;
} lamb_matrix;

/* A list of matrices that are worked on together, with their workspace: about
 * 4 bytes per element and 4 per entry of the short sides' squares (12 for matrices
 * at least twice as long as wide in lists with much to do), twice that with
 * LAMB_NS_SPLIT. Calls share the workspace: one on another stream than the plan's last
 * call waits for that one's work. Replays of a captured call are not seen; the caller
 * orders them among themselves and with other calls. Not thread-safe. */
typedef struct lamb_ns_plan lamb_ns_plan;

/*
 * `matrices` (host) has n >= 1 entries; in_dtype and out_dtype are
 * LAMB_DTYPE_F32 or LAMB_DTYPE_BF16; precision is a lamb_ns_precision.
 */
LAMB_API lamb_status lamb_ortho_plan_create(const lamb_matrix *matrices, int32_t n,
                                            int32_t in_dtype, int32_t out_dtype,
                                            int32_t precision, lamb_ns_plan **out);

/* Every out becomes the iteration's result for its in. A matrix that holds a NaN
 * or an infinity becomes NaN; the others are not touched by it. */
LAMB_API lamb_status lamb_orthogonalize(lamb_ns_plan *plan, const lamb_ns_params *params,
                                        void *stream);

/*
 * One matrix of a Muon step: contiguous, row-major. x fp32 parameters and m fp32
 * momentum are updated in place, g (fp32 or bf16, one type per plan) is read. The
 * conventions of lamb_tensor hold, and its alignment (16 bytes).
 */
typedef struct lamb_muon_tensor {
    float *x;
    const void *g;
    float *m;
    int64_t rows, cols;
    int32_t wd;       /* 1: weight decay applies to this matrix */
    int32_t reserved; /* must be 0 */
} lamb_muon_tensor;

LAMB_API lamb_status lamb_muon_plan_create(const lamb_muon_tensor *tensors, int32_t n,
                                           int32_t g_dtype, int32_t precision,
                                           lamb_ns_plan **out);

/* The factor s of the update: LAMB_MUON_RMS 0.2 sqrt(max(rows, cols)), which gives
 * the update an Adam step's root mean square; LAMB_MUON_SPECTRAL
 * sqrt(max(1, rows / cols)); LAMB_MUON_UNIT 1. */
typedef enum lamb_muon_scale {
    LAMB_MUON_RMS = 0,
    LAMB_MUON_SPECTRAL = 1,
    LAMB_MUON_UNIT = 2
} lamb_muon_scale;

typedef struct lamb_muon_hparams {
    lamb_ns_params ns;
    float lr;            /* >= 0                                                 */
    double momentum;     /* in [0, 1); 1 - momentum is taken of this, where that of
                            a float near 0.95 would be 2.4e-7 off             */
    float weight_decay;  /* >= 0, decoupled: x <- (1 - lr weight_decay) x first   */
    float grad_scale;    /* > 0: every gradient element is multiplied by it       */
    int32_t nesterov;    /* 0 or 1                                               */
    int32_t scale;       /* a lamb_muon_scale                                    */
    int32_t skip_nonfinite; /* 1: a step whose scaled gradient holds a NaN or an
                               infinity anywhere changes nothing                 */
    int32_t reserved;    /* must be 0                                            */
} lamb_muon_hparams;

/* lr 1e-3, momentum 0.95, Nesterov, no decay, LAMB_MUON_RMS, grad_scale 1. */
LAMB_API lamb_status lamb_muon_hparams_init(lamb_muon_hparams *hp);

/*
 * g' = grad_scale g;  m <- momentum m + (1 - momentum) g';
 * u = momentum m + (1 - momentum) g' (Nesterov) or m;  O = the iteration's result for u;
 * x <- (1 - lr weight_decay wd) x - lr s O.
 * nonfinite_out (device int32, may be NULL) receives 1 when skip_nonfinite held the
 * step back, else 0.
 */
LAMB_API lamb_status lamb_muon_step(lamb_ns_plan *plan, const lamb_muon_hparams *hp, void *stream,
                                    int32_t *nonfinite_out);

/* Frees either kind of plan; NULL is fine. Waits for the device. */
LAMB_API lamb_status lamb_ns_plan_destroy(lamb_ns_plan *plan);

/*
 * Softmax cross entropy of hidden states against a vocabulary table:
 * logits = hidden table^T, loss_i = logsumexp(logits_i) - logits_i[target_i].
 * hidden [tokens][dim] and table [vocab][dim] are bfloat16, rows `*_stride` elements
 * apart (>= dim), 2-byte aligned. Every call copies the rows of hidden whose tokens count
 * to the workspace. The table is read in place where its rows are 16-byte aligned and at
 * most 2^21 elements apart and dim is a multiple of 8; else it is copied too.
 * targets: LAMB_DTYPE_I32 or _I64. A token whose target is ignore_index does not
 * count: its loss and gradient are 0 and nothing that its row holds reaches any
 * result. Any other target outside [0, vocab) makes that token's loss and lse NaN, and
 * with them the mean and the gradients.
 * tokens 0 to 2^24, vocab 1 to 2^24, dim 1 to 2^16, strides at most 2^36.
 */
typedef struct lamb_xent {
    const void *hidden;
    const void *table;
    const void *targets;
    int64_t hidden_stride, table_stride;
    int64_t tokens, vocab, dim;
    int64_t ignore_index;
    int32_t target_dtype;
    int32_t reserved; /* must be 0 */
} lamb_xent;

/* Bytes of device workspace (256-byte aligned) that a forward and a backward call need;
 * host only. For T tokens, V words and rows of D columns (dim rounded up to 8), at most,
 * beside a few KiB of alignment:
 *  both      (2 D + 8) T for the rows that count, packed together, and 2 D V for the table
 *            where it is copied
 *  forward   8 T for every tile of 64 words, and 4 T (large calls take tiles of 128 or 256
 *            words: 1.6 GiB for 2^20 tokens against 50257)
 *  backward  160 MiB, or 512 T where that is more (from 327,681 tokens on), for a piece of
 *            the vocabulary's softmax; 4 D T for the hidden states' gradient in fp32,
 *            whether it is asked for or not, and 128 MiB of parts of it where workgroups
 *            share the sums of few rows; from 32,769 tokens on 10,240 D for a piece of the
 *            table's gradient
 */
LAMB_API lamb_status lamb_xent_workspace(const lamb_xent *xent, size_t *forward_bytes,
                                         size_t *backward_bytes);

/*
 * loss and lse: device float[tokens], fp32 (lse is what the backward needs). mean:
 * device float, the sum of the losses over the number of tokens that count (0 when
 * none does), or NULL.
 */
LAMB_API lamb_status lamb_xent_forward(const lamb_xent *xent, float *loss, float *lse, float *mean,
                                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Gradients of grad_scale grad_loss times the mean (`mean` 1) or the sum (0) of the
 * losses, given the forward's lse. grad_loss: device float, or NULL for 1.
 * grad_hidden: bfloat16 [tokens][dim], or NULL. grad_table: [vocab][dim] of
 * grad_table_dtype (LAMB_DTYPE_F32 or _BF16), written, or added to (`add_table` 1);
 * NULL for none.
 * Both are sums of the softmax less one at the target, times rows. For 16-bit gradients
 * it is rounded to bfloat16, each entry by itself: as 2-norms they are 1.7e-3 off, by
 * their own rounding, to 2.5e-3, where the terms are of one size and few. For an fp32
 * grad_table it is held in 16 bits (2^-16 of each entry at most), for a product more. lse
 * as an fp32 number adds 2^-24 of the largest logit to either.
 */
typedef struct lamb_xent_grads {
    const float *grad_loss;
    void *grad_hidden;
    void *grad_table;
    int64_t grad_hidden_stride, grad_table_stride;
    int32_t grad_table_dtype;
    int32_t add_table;
    int32_t mean;
    float grad_scale;
} lamb_xent_grads;

LAMB_API lamb_status lamb_xent_backward(const lamb_xent *xent, const float *lse,
                                        const lamb_xent_grads *grads, void *workspace,
                                        size_t workspace_bytes, void *stream);

/*
 * Rows of a token table: out[i] = scale table[ids[i]]. table [vocab][dim] and out
 * [tokens][dim] are float32 or bfloat16 each, rows `*_stride` elements apart (>= dim;
 * out's rows do not overlap), aligned to their elements. ids: LAMB_DTYPE_I32 or _I64.
 * The row of an id outside [0, vocab) becomes NaN. tokens 0 to 2^24, vocab 1 to 2^24,
 * dim 1 to 2^16, strides at most 2^36.
 */
typedef struct lamb_embed {
    const void *ids;
    int64_t tokens, vocab, dim;
    int32_t id_dtype;
    float scale;
} lamb_embed;

LAMB_API lamb_status lamb_embed_forward(const lamb_embed *embed, const void *table,
                                        int64_t table_stride, int32_t table_dtype, void *out,
                                        int64_t out_stride, int32_t out_dtype, void *stream);

/*
 * The table's gradient: grad_table[v] = (or, with `add` 1, +=) scale times the sum of
 * grad_out[i] over the tokens with ids[i] = v, in the tokens' order and in fp32, at most
 * 16 tokens, then 64 such sums at a time: the same inputs give the same bits. Tokens whose
 * id is outside the table or equals padding_id (-1 for none) add nothing. Without `add`
 * every row is written; with it, only rows that tokens name are touched.
 * lamb_embed_workspace gives the device workspace's bytes (256-byte aligned; host only).
 */
LAMB_API lamb_status lamb_embed_workspace(const lamb_embed *embed, size_t *bytes);

LAMB_API lamb_status lamb_embed_backward(const lamb_embed *embed, const void *grad_out,
                                         int64_t grad_out_stride, int32_t grad_out_dtype,
                                         void *grad_table, int64_t grad_table_stride,
                                         int32_t grad_table_dtype, int64_t padding_id, int32_t add,
                                         void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* LAMB_OPS_H */
