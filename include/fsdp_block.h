/*
 * fsdp_block.h - the operators a training step runs between the copy-out of a
 * bucket's parameters (fsdp_ag_unpack) and the copy-in of their gradients
 * (fsdp_rs_pack), on an AMD Instinct MI355X (gfx950): the norms before and
 * after a block, the block's matrix products, and a distillation loss, each
 * with its gradient.  They read the parameters where the copy-out wrote them
 * and write the gradients where the copy-in reads them.
 *
 * Conventions for every call (those of fsdp_bucket.h, and):
 *   - Device pointers are HIP device memory on the current device.  The
 *     caller owns every buffer.  The calls allocate nothing and never
 *     synchronise; they enqueue a fixed number of kernels on `stream`.
 *   - All arguments are validated on the host before any HIP call; on any
 *     error nothing is enqueued and no output is touched.
 *   - A matrix is row-major with its columns contiguous; `*_stride` is the
 *     distance of its rows in elements (at least the row's length; any value
 *     where there is one row or none).  Vectors are contiguous.  Pointers need
 *     element alignment only; kernels take 16 bytes at a time off the 16-byte
 *     grid too, unless a comment says otherwise.
 *   - A pointer may be NULL where a comment says "or NULL", or where the
 *     matrix has no elements.
 *   - Outputs must not overlap inputs or each other, except that an output may
 *     BE an input (same pointer, stride and type) where a comment says so.  An
 *     input that other rows or columns read too (a weight, a bias, a gate, the
 *     factors of a product) may not lie there even then.
 *     Matrices of one row stride may interleave (column slices of one buffer).
 *   - Sums, statistics and products are held in fp32; each output is rounded
 *     once, to nearest even, unless a comment says otherwise.  Results do not
 *     depend on timing, the same call gives the same bits: sums are joined in a
 *     fixed order, and nothing but counts of equal ids is atomic.
 *   - A call that needs scratch memory takes `workspace`, of at least the
 *     bytes its *_workspace query returns for the same arguments, 256-byte
 *     aligned; what it holds before the call does not matter, and it is free
 *     again once the call's kernels have run.  NULL if the query says 0.
 */
#ifndef FSDP_BLOCK_H
#define FSDP_BLOCK_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "fsdp_bucket.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Detail of this thread's last error in this library (never NULL). */
const char* fsdp_block_last_error(void);

/* ------------------------------------------------------------------ norms
 *
 * For every token t, with rms(v) = v / sqrt(mean(v^2) + eps):
 *
 *     n = rms(branch) * post_weight          (branch itself without post_weight)
 *     y = residual_scale * x + branch_scale * gate * n
 *     h = rms(y) * pre_weight
 *
 * the norm after a block with its gate and the residual add, and the norm
 * before the next block.  Without a branch, y = residual_scale * x.  h is
 * computed from y before y is rounded.
 *
 * gate has gate_rows rows; token t takes row t / (tokens / gate_rows):
 * gate_rows = 1 is one vector for all, the number of sequences a row for each
 * sequence, tokens a row for each token.  (Without tokens the gradient takes at most
 * 60000 rows.)
 */
#define FSDP_NORM_MAX_HIDDEN 16384

typedef struct fsdp_norm_args {
    int64_t tokens;                /* >= 0 */
    int64_t hidden;                /* 1 .. FSDP_NORM_MAX_HIDDEN */
    int64_t gate_rows;             /* 0 without a gate, else a divisor of tokens */
    fsdp_dtype stream_dtype;       /* x and y: the block's type, or F32 */
    fsdp_dtype block_dtype;        /* branch, h and gate */
    fsdp_dtype weight_dtype;       /* both weights: the block's type, or F32 */
    float eps, residual_scale, branch_scale;     /* eps >= 0 */
    const void* x;
    const void* branch;            /* or NULL */
    const void* post_weight;       /* [hidden] or NULL; needs a branch */
    const void* gate;              /* [gate_rows, hidden], rows contiguous, or NULL; needs a branch */
    const void* pre_weight;        /* [hidden], or NULL without h */
    void* y;                       /* may be x; NULL if only h is wanted */
    void* h;                       /* may be branch; NULL if only y is wanted */
    int64_t x_stride, branch_stride, y_stride, h_stride;
} fsdp_norm_args;

/* One kernel (none without tokens). */
fsdp_status fsdp_block_norm(const fsdp_norm_args* args, hipStream_t stream);

/*
 * The gradient.  y is what fsdp_block_norm wrote (rounded); both row
 * statistics are computed again from y and branch, nothing else is kept.
 * With dy the gradient that reaches y from what follows it (NULL: zero) and
 * dh that of h (NULL: zero):
 *
 *     g  = dy + grad of rms(y) * pre_weight at dh
 *     dx = residual_scale * g
 *     dbranch, dpost_weight, dgate from branch_scale * g
 *     dpre_weight = sum over tokens of dh * rms(y)
 *
 * Any output may be NULL.  dgate sums over the tokens of its row, the weight
 * gradients over all tokens (zeros without tokens).
 */
typedef struct fsdp_norm_grad_args {
    int64_t tokens, hidden, gate_rows;
    fsdp_dtype stream_dtype;       /* y, dy and dx */
    fsdp_dtype block_dtype;        /* dh, branch, gate, dbranch and dgate */
    fsdp_dtype weight_dtype;       /* the weights and their gradients */
    float eps, residual_scale, branch_scale;
    const void* y;                 /* needed with dh */
    const void* dy;                /* or NULL */
    const void* dh;                /* or NULL; needs pre_weight */
    const void* branch;            /* or NULL */
    const void* post_weight;       /* or NULL; needs a branch */
    const void* gate;              /* or NULL; needs a branch */
    const void* pre_weight;        /* or NULL; needs dh */
    void* dx;                      /* may be dy */
    void* dbranch;                 /* may be branch or dh; needs a branch */
    void* dpre_weight;             /* needs pre_weight */
    void* dpost_weight;            /* needs post_weight */
    void* dgate;                   /* [gate_rows, hidden]; needs a gate */
    int64_t y_stride, dy_stride, dh_stride, branch_stride, dx_stride, dbranch_stride;
} fsdp_norm_grad_args;

fsdp_status fsdp_block_norm_grad_workspace(const fsdp_norm_grad_args* args, int64_t* bytes);
/* One kernel, and one more where a column sum is wanted. */
fsdp_status fsdp_block_norm_grad(const fsdp_norm_grad_args* args, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream);

/* ------------------------------------------------------------------ linear
 *
 *     z   = x weight^T + bias
 *     out = act(z) * times + residual
 *
 * x [m, k], weight [n, k] (a parameter as the copy-out leaves it), bias [n],
 * times, residual, pre and out [m, n], all of one type.  `pre` keeps z,
 * rounded, for the gradient; out is computed from z before that.  Activations
 * are off by some 12 units of 2^-24 of themselves in fp32 (GELU's tanh form by 4 of
 * its argument more in its tail), by up to 7e-6 before the rounding to 16 bits; what
 * takes an exponential below 2^-126 is 0.
 *
 * Sizes are at most 2^30, with 2^22 tiles of 64 x 64 in every matrix.  With more than
 * four rows of x, 64 rows of x and of weight (fp32: 64 and 128; all, if there are fewer)
 * must lie within 2^31 bytes, at rows of k in whole 128-byte lines: k up to 17 million in
 * 16 bits, 4.2 million in fp32.  The gradient's products ask the same of n for dz, and of k
 * and n 17 million.  Else FSDP_ERR_OVERFLOW.
 */
typedef int32_t fsdp_activation;
enum {
    FSDP_ACT_NONE = 0,
    FSDP_ACT_RELU = 1,
    FSDP_ACT_SILU = 2,             /* z / (1 + exp(-z)) */
    FSDP_ACT_GELU = 3,             /* z * Phi(z), Phi the normal distribution */
    FSDP_ACT_GELU_TANH = 4         /* its tanh form */
};

typedef struct fsdp_linear_args {
    int64_t m, n, k;               /* m, n >= 0, k >= 1 */
    fsdp_dtype dtype;
    fsdp_activation activation;
    const void* x;
    const void* weight;
    const void* bias;              /* or NULL */
    const void* times;             /* or NULL */
    const void* residual;          /* or NULL */
    void* pre;                     /* or NULL */
    void* out;                     /* may be times or residual */
    int64_t x_stride, weight_stride, times_stride, residual_stride, pre_stride, out_stride;
} fsdp_linear_args;

fsdp_status fsdp_block_linear_workspace(const fsdp_linear_args* args, int64_t* bytes);
/* One kernel; one before it where x or weight lies off the 16-byte grid (up to
 * four rows of x excepted), one after it where few tiles split the sum over k,
 * or many leave a last round of few.  None where out has no elements. */
fsdp_status fsdp_block_linear(const fsdp_linear_args* args, void* workspace, int64_t workspace_bytes,
                              hipStream_t stream);

/*
 * The gradient, from dout [m, n]:
 *
 *     dz = dout * times * act'(z)      dtimes  = dout * act(z)
 *     dx = dz weight [m, k]            dweight = dz^T x [n, k]
 *     dbias = sum of dz over the rows  (the residual's gradient is dout)
 *
 * Any output may be NULL.  z comes from `pre`, needed with an activation and
 * for dtimes.  dz enters the two products rounded to the type (the matrix
 * cores take 16-bit factors; with neither activation nor times it is dout
 * itself); dbias sums it before that.  dweight and dbias are zeros when m is 0.
 */
typedef struct fsdp_linear_grad_args {
    int64_t m, n, k;
    fsdp_dtype dtype;
    fsdp_activation activation;
    const void* dout;
    const void* x;                 /* or NULL without dweight */
    const void* weight;            /* or NULL without dx */
    const void* pre;               /* or NULL */
    const void* times;             /* or NULL */
    void* dx;
    void* dweight;
    void* dbias;                   /* [n] */
    void* dtimes;                  /* may be times; needs times */
    int64_t dout_stride, x_stride, weight_stride, pre_stride, times_stride;
    int64_t dx_stride, dweight_stride, dtimes_stride;
} fsdp_linear_grad_args;

fsdp_status fsdp_block_linear_grad_workspace(const fsdp_linear_grad_args* args, int64_t* bytes);
/* At most one kernel for dz and its sums, one to join the sums, and for each
 * product as many as fsdp_block_linear. */
fsdp_status fsdp_block_linear_grad(const fsdp_linear_grad_args* args, void* workspace, int64_t workspace_bytes,
                                   hipStream_t stream);

/* ------------------------------------------------------------------ distillation
 *
 * Distillation from a teacher's top logits.  For every token, with the
 * student's logits s [vocab] and the teacher's v [top] at the vocabulary
 * places ids [top], q = softmax(s / tau) and
 *
 *     p_k = exp(v_k / tau - L),  L = teacher_lse, or the logsumexp of the row's
 *                                valid v_k / tau without it (then sum p = 1)
 *     loss = tau^2 * sum_k p_k * (log p_k - log q[ids_k])
 *     dlogits_j = dloss * tau * (q_j * sum_k p_k - sum of p_k with ids_k = j)
 *
 * An entry with ids_k < 0 is not valid: v_k is not used.  A row without a
 * valid entry, or whose valid v_k are all -inf, has loss 0, lse 0 and gradient
 * 0, whatever its logits hold.  p_k = 0 contributes 0.  A row with an id of
 * vocab or more has loss and gradient NaN.  A dloss of 0 gives a gradient of 0.
 * Masked logits may be -inf or any finite value, over a part of a row or all of it
 * (q and p are then uniform).  A saved lse is an fp32 value: the gradient from it is
 * off by exp of its rounding, so that a row of logits that are all at such a mask
 * has its gradient from fsdp_block_distill only.
 */
#define FSDP_DISTILL_MAX_TOP 1024

typedef struct fsdp_distill_args {
    int64_t tokens;                /* >= 0 */
    int64_t vocab;                 /* 1 .. 2^31 - 1 - 2^16 */
    int64_t top;                   /* 1 .. FSDP_DISTILL_MAX_TOP */
    fsdp_dtype dtype;              /* logits and dlogits */
    fsdp_dtype teacher_dtype;
    int32_t ids_64;                /* ids are int64_t, else int32_t */
    float temperature;             /* tau > 0, finite */
    const void* logits;            /* [tokens, vocab] */
    const void* teacher;           /* [tokens, top], rows contiguous */
    const void* ids;               /* [tokens, top], rows contiguous */
    const float* teacher_lse;      /* [tokens] or NULL */
    const float* dloss;            /* [tokens]; needed with dlogits */
    float* loss;                   /* [tokens], or NULL */
    float* lse;                    /* [tokens]: logsumexp of s / tau.  fsdp_block_distill writes it (or NULL),
                                      fsdp_block_distill_grad reads it */
    void* dlogits;                 /* [tokens, vocab], may be logits */
    int64_t logits_stride, dlogits_stride;
} fsdp_distill_args;

/* The loss, lse, and with dlogits the gradient in the same pass.  One kernel. */
fsdp_status fsdp_block_distill(const fsdp_distill_args* args, hipStream_t stream);
/* The gradient from the lse that fsdp_block_distill wrote (loss is not used).  One kernel. */
fsdp_status fsdp_block_distill_grad(const fsdp_distill_args* args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif  /* FSDP_BLOCK_H */
