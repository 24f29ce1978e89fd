/*
 * fsdp_step.h - more of what a training step runs between the copy-out of a
 * bucket's parameters and the copy-in of their gradients, on an AMD Instinct
 * MI355X (gfx950): a gated feed-forward's projections with their activation and
 * product, matrices kept in 8 bits for the backward pass, and a clipped policy
 * loss with its KL term, each with its gradient.
 *
 * The conventions are those of fsdp_block.h (buffers, streams, strides, what may
 * overlap, workspaces, roundings, fixed results).  The library links
 * libfsdp_block.so, whose fsdp_block_last_error holds the detail of this
 * thread's last error in either.
 *
 * A matrix in 8 bits.  32 neighbouring columns of a row are a group (the last
 * one of a row may be shorter).  With M the largest magnitude of a group,
 *
 *     e = the least integer >= -126 with M / 2^e rounding to 127 or less
 *     codes = v / 2^e, rounded to the nearest integer, ties to even
 *     scale byte = e + 127             (1 .. 249)
 *
 * and it stands for codes * 2^e.  A group that holds an infinity or a NaN has the
 * byte 255 and stands for NaN.  So codes [rows, cols] are int8 and scales
 * [rows, ceil(cols / 32)] uint8, each with a row stride of its own.  The scale is
 * a power of two because what a group stands for is then exact in bf16, fp16 and
 * fp32, between the ends of their ranges: the matrix cores take it with no further
 * rounding.  A step is at most 2^-6 of the group's largest magnitude, a value is off by
 * half of one.
 *
 * At the ends: what passes a type's range is infinite in it, and the largest values of a
 * group may round up to a power of two past it (M from 65280 on stands for 65536, infinite
 * in fp16; from 255 * 2^120 on for 2^128, infinite in every type).  A group with steps
 * below 2^-24, of M below 2^-18, is rounded a second time where it is read as fp16, to
 * multiples of 2^-24, unless it was saved from fp16.  (fsdp_step_gated saves its sums in
 * 32 bits.)
 */
#ifndef FSDP_STEP_H
#define FSDP_STEP_H

#include "fsdp_block.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FSDP_STEP_GROUP 32

/* ------------------------------------------------------------------ 8 bits */

typedef struct fsdp_step_save_args {
    int64_t rows, cols;            /* >= 0; rows below 2^31, cols at most 2^30 */
    fsdp_dtype dtype;              /* of x */
    const void* x;                 /* [rows, cols] */
    void* codes;
    void* scales;
    int64_t x_stride, codes_stride, scales_stride;
} fsdp_step_save_args;

/* x to 8 bits.  One kernel, none without elements. */
fsdp_status fsdp_step_save(const fsdp_step_save_args* args, hipStream_t stream);

typedef struct fsdp_step_restore_args {
    int64_t rows, cols;
    fsdp_dtype dtype;              /* of x */
    const void* codes;
    const void* scales;
    void* x;                       /* [rows, cols] */
    int64_t codes_stride, scales_stride, x_stride;
} fsdp_step_restore_args;

/* What a matrix in 8 bits stands for.  One kernel, none without elements. */
fsdp_status fsdp_step_restore(const fsdp_step_restore_args* args, hipStream_t stream);

/* ------------------------------------------------------------------ gated feed-forward
 *
 *     g = x gate_weight^T      u = x up_weight^T      out = act(g) * u
 *
 * x [m, k], both weights [n, k], out [m, n], all of one type; activations as in
 * fsdp_block.h.  gate and up keep g and u for the gradient: both or neither, in
 * the type, or in 8 bits where their scales are given.  out, and the 8 bits, are
 * computed from g and u before these are rounded.
 *
 * Sizes are below 2^29, with 2^22 tiles of 64 x 64 in every matrix, both weights
 * counted as one of 2 n rows.  64 rows of x and 128 of a weight must lie within 2^31
 * bytes, at rows of k in whole 128-byte lines, but for up to four rows of x, which go
 * without tiles where n is below 2^26 and nothing is kept in 8 bits.  Else
 * FSDP_ERR_OVERFLOW.
 */
typedef struct fsdp_step_gated_args {
    int64_t m, n, k;               /* m, n >= 0, k >= 1 */
    fsdp_dtype dtype;
    fsdp_activation activation;
    const void* x;
    const void* gate_weight;
    const void* up_weight;
    void* gate;                    /* or NULL */
    void* gate_scales;             /* or NULL: gate is of the type */
    void* up;                      /* or NULL, as gate */
    void* up_scales;               /* or NULL, as gate_scales */
    void* out;
    int64_t x_stride, gate_weight_stride, up_weight_stride;
    int64_t gate_stride, gate_scales_stride, up_stride, up_scales_stride, out_stride;
} fsdp_step_gated_args;

fsdp_status fsdp_step_gated_workspace(const fsdp_step_gated_args* args, int64_t* bytes);
/* One kernel; for tiles one before it where x or a weight lies off the 16-byte grid, and
 * one after it where few tiles split the sum over k, or many leave a last round of
 * few.  None where out has no elements. */
fsdp_status fsdp_step_gated(const fsdp_step_gated_args* args, void* workspace, int64_t workspace_bytes,
                            hipStream_t stream);

/*
 * The gradient, from dout [m, n] and what gate and up keep:
 *
 *     dg = dout * u * act'(g)                 du = dout * act(g)
 *     dx = dg gate_weight + du up_weight      out = act(g) * u, again
 *     dgate_weight = dg^T x                   dup_weight = du^T x
 *
 * Any output may be NULL.  gate, up and x are of the type, or in 8 bits where
 * their scales are given (gate and up alike).  dg and du enter the products rounded
 * to the type.  The weights' gradients are zeros when m is 0.
 */
typedef struct fsdp_step_gated_grad_args {
    int64_t m, n, k;
    fsdp_dtype dtype;
    fsdp_activation activation;
    const void* dout;              /* with any output */
    const void* x;                 /* or NULL without the weights' gradients */
    const void* x_scales;          /* or NULL */
    const void* gate_weight;       /* or NULL without dx */
    const void* up_weight;         /* or NULL without dx */
    const void* gate;
    const void* gate_scales;       /* or NULL */
    const void* up;
    const void* up_scales;         /* or NULL */
    void* out;                     /* may be dout */
    void* dx;
    void* dgate_weight;            /* both weights' gradients, or neither */
    void* dup_weight;
    int64_t dout_stride, x_stride, x_scales_stride, gate_weight_stride, up_weight_stride;
    int64_t gate_stride, gate_scales_stride, up_stride, up_scales_stride;
    int64_t out_stride, dx_stride, dgate_weight_stride, dup_weight_stride;
} fsdp_step_gated_grad_args;

fsdp_status fsdp_step_gated_grad_workspace(const fsdp_step_gated_grad_args* args, int64_t* bytes);
/* One kernel for dg, du and out; one that restores an x in 8 bits; for each of dx and
 * the weights' gradients as many as fsdp_step_gated (one before it at most). */
fsdp_status fsdp_step_gated_grad(const fsdp_step_gated_grad_args* args, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream);

/* ------------------------------------------------------------------ linear, from 8 bits
 *
 * The gradient of fsdp_block_linear (its formulas and arguments) with x, `pre` or both
 * in 8 bits, where their scales are given; with neither, fsdp_block_linear_grad
 * does the same work.
 */
typedef struct fsdp_step_linear_grad_args {
    int64_t m, n, k;
    fsdp_dtype dtype;
    fsdp_activation activation;
    const void* dout;
    const void* x;                 /* or NULL without dweight */
    const void* x_scales;          /* or NULL */
    const void* weight;            /* or NULL without dx */
    const void* pre;               /* or NULL */
    const void* pre_scales;        /* or NULL */
    const void* times;             /* or NULL */
    void* dx;
    void* dweight;
    void* dbias;                   /* [n] */
    void* dtimes;                  /* may be times; needs times */
    int64_t dout_stride, x_stride, x_scales_stride, weight_stride, pre_stride, pre_scales_stride, times_stride;
    int64_t dx_stride, dweight_stride, dtimes_stride;
} fsdp_step_linear_grad_args;

fsdp_status fsdp_step_linear_grad_workspace(const fsdp_step_linear_grad_args* args, int64_t* bytes);
fsdp_status fsdp_step_linear_grad(const fsdp_step_linear_grad_args* args, void* workspace, int64_t workspace_bytes,
                                  hipStream_t stream);

/* ------------------------------------------------------------------ policy loss
 *
 * The clipped policy loss of a sampled token with its KL term.  For every token,
 * with the logits s [vocab], the action a that was taken, its log probability `old`
 * under the policy that took it, its advantage A, and q = softmax(s / tau):
 *
 *     logp = log q[a]          r = exp(logp - old)
 *     loss = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *            + kl_weight * (exp(d) - d - 1),      d = ref - logp
 *     slope = (r A <= clip(r) A ? -r A : 0) + kl_weight * (1 - exp(d))
 *     dlogits_j = dloss * slope / tau * ((j = a) - q_j)
 *
 * `slope` is the loss's with respect to logp.  ref is the action's log probability
 * under a reference policy; without ref_logp there is no KL term.  A token with
 * a < 0 (a prompt's, or padding) has loss, logp, lse and gradient 0, whatever its
 * other values are; one with a of vocab or more NaN.  A dloss of 0 gives a
 * gradient of 0.  Masked logits may be -inf or any finite value; a row whose logits
 * are all -inf has no distribution: NaN.  An advantage of 0 adds nothing, whatever
 * r is.  Differences of logarithms are formed in 64 bits, and dloss * slope / tau is then
 * an fp32 value: a row in which it passes their range has a gradient that is not finite.
 *
 * A saved lse is an fp32 value, and below 2^14 the gradient from it takes it as it is:
 * q and r are off by exp of its rounding, 2^-24 |lse|, at most 2^-11 of themselves.
 * From 2^14 on (a small tau, a row far from 0 or all at a mask's finite value) that
 * gradient takes the row's own maximum and sum instead, and is as exact as the one of
 * fsdp_step_policy.
 */
typedef struct fsdp_step_policy_args {
    int64_t tokens;                /* >= 0 */
    int64_t vocab;                 /* 1 .. 2^31 - 1 - 2^16 */
    fsdp_dtype dtype;              /* logits and dlogits */
    int32_t actions_64;            /* actions are int64_t, else int32_t */
    float clip_low;                /* 0 .. 1 */
    float clip_high;               /* >= 0, may be infinite */
    float kl_weight;               /* finite; needs ref_logp unless 0 */
    float temperature;             /* tau >= 2^-126, finite */
    const void* logits;            /* [tokens, vocab] */
    const void* actions;           /* [tokens] */
    const float* old_logp;         /* [tokens] */
    const float* advantages;       /* [tokens] */
    const float* ref_logp;         /* [tokens] or NULL */
    const float* dloss;            /* [tokens]; needed with dlogits */
    float* loss;                   /* [tokens] or NULL */
    float* logp;                   /* [tokens] or NULL */
    float* lse;                    /* [tokens]: logsumexp of s / tau.  fsdp_step_policy writes it (or NULL),
                                      fsdp_step_policy_grad reads it */
    void* dlogits;                 /* [tokens, vocab], may be logits */
    int64_t logits_stride, dlogits_stride;
} fsdp_step_policy_args;

/* The loss, logp, lse, and with dlogits the gradient in the same pass.  One kernel. */
fsdp_status fsdp_step_policy(const fsdp_step_policy_args* args, hipStream_t stream);
/* The gradient from the lse that fsdp_step_policy wrote for these logits (loss and logp are not used).  One kernel. */
fsdp_status fsdp_step_policy_grad(const fsdp_step_policy_args* args, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif  /* FSDP_STEP_H */
