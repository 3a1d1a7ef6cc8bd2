/*
 * mergecomp_step.h -- C ABI of the operators on either side of a training step's exchange of gradients, in the same
 * library as mergecomp.h.
 *
 * After the exchange, over a model's list of tensors (the ones whose gradients mc_decompress_sum has written):
 *     mc_grad_norm    global 2-norm and the clipping coefficient that follows from it
 *     mc_grad_clip    the same, and the clipped gradients
 *     mc_adamw        AdamW update with the coefficient taken from device memory
 * Before it, where back-propagation starts, over rows of logits:
 *     mc_token_logp   log-probabilities of given tokens
 *     mc_policy_loss  clipped policy loss with a KL term, and its gradient, in one call
 *
 * Conventions
 *   - those of mergecomp.h: pointers are "host" or "device" as stated, calls only enqueue kernels on the caller's stream
 *     (void* = hipStream_t), allocate nothing, never synchronise and read nothing back; all calls on one handle must be
 *     issued in stream order, since its scratch is shared between them.  0 or a negative mc_status; no call throws or aborts.
 *   - A handle belongs to the device that was current when it was made: its calls take memory of that device and a stream of it (NULL:
 *     the current device's, which has to be that one).
 *   - Arithmetic is binary32; sums over tensors and over rows are binary64.  Sums are taken in an order that depends on sizes, on where
 *     rows and tensors begin in a cache line, and on the device alone: the same call gives the same bits.  Values of 16
 *     bits are widened when they are read and rounded once, to nearest even, when they are written.
 *   - What a call writes may not lie over anything else that it writes or reads, except where it is said below.
 *   - Tensors may start at any address that is a multiple of their element size; multiples of 16 bytes are fastest.
 */
#ifndef MERGECOMP_STEP_H
#define MERGECOMP_STEP_H

#include "mergecomp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MC_DTYPE_NONE = -1,
    MC_DTYPE_F32 = 0,
    MC_DTYPE_BF16 = 1,
    MC_DTYPE_F16 = 2
} mc_dtype;

/* ---- a model's list of tensors ------------------------------------------------------------------------------- */
typedef struct mc_step mc_step;

/* The lists that a handle knows, each one tensor for every tensor of the model. */
typedef enum {
    MC_LIST_GRADS = 0,       /* grad_dtype                                                                         */
    MC_LIST_CLIPPED = 1,     /* grad_dtype; what mc_grad_clip writes.  Not bound, or
                                bound to the same addresses: the gradients themselves                              */
    MC_LIST_PARAMS = 2,      /* fp32 weights                                                                       */
    MC_LIST_EXP_AVG = 3,     /* fp32 first moments                                                                 */
    MC_LIST_EXP_AVG_SQ = 4,  /* fp32 second moments                                                                */
    MC_LIST_MODEL = 5,       /* model_dtype; what forward and backward passes read, written by mc_adamw              */
    MC_LISTS = 6
} mc_list;

/*
 * A handle for one list of tensors on the current HIP device.
 *   numel        host, n_tensors sizes in elements (>= 0), copied
 *   grad_dtype   mc_dtype of gradients and clipped gradients
 *   model_dtype  mc_dtype of the model's copy of the weights: MC_DTYPE_BF16, MC_DTYPE_F16, or MC_DTYPE_NONE for no copy
 *   no_decay     host, n_tensors bytes, not 0 where mc_adamw's weight decay leaves a tensor out (biases, norms); may be NULL
 * Device memory: 16 bytes per 4096 elements of a tensor, 48 per tensor, about 20 KB besides.
 * Errors: MC_ERR_INVALID_ARG (null, n_tensors < 1, negative size, unknown type), MC_ERR_RANGE (a tensor of 2^39
 * elements or more, more than 2^27 blocks of 4096 elements in all), MC_ERR_ALLOC, MC_ERR_DEVICE.
 */
int mc_step_create(mc_step **out, const int64_t *numel, int32_t n_tensors, int32_t grad_dtype, int32_t model_dtype,
                   const uint8_t *no_decay);
int mc_step_destroy(mc_step *h);

/*
 * Where the tensors of a list lie: used by the calls issued afterwards, until the list is bound again.
 *   ptrs   host array of n_tensors DEVICE pointers (copied; null only for a tensor without elements)
 * One or a few small launches; a program whose gradients stay in place binds them once.
 */
int mc_step_bind(mc_step *h, int32_t list, const void *const *ptrs, void *stream);

/*
 * norm = scale * sqrt(sum of the squares of all elements of all gradients)
 * coef = scale * min(1, max_norm / (norm + 1e-6)), or 0 if a gradient holds an infinity or a NaN
 *   scale      what a gradient is multiplied by before anything else (1 / loss scale, 1 / accumulated steps); finite, > 0
 *   max_norm   > 0; infinity: nothing is clipped
 *   out        device, two floats: norm, coef
 * Squares are summed in binary64, so that neither large nor small gradients are lost.  A finite norm beyond binary32 is
 * written as infinity; its coef follows from the norm as it is, rounded to binary32: below 2^-126 it has fewer digits, below 2^-150
 * it is 0 and so stands for a step that is left out.
 */
int mc_grad_norm(mc_step *h, float scale, float max_norm, float *out, void *stream);

/* mc_grad_norm, and every gradient times coef into MC_LIST_CLIPPED, which may be the gradients themselves but may not
 * overlap them otherwise.  Where coef is 0 the result is 0, also for infinities and NaN. */
int mc_grad_clip(mc_step *h, float scale, float max_norm, float *out, void *stream);

/*
 * One AdamW update, with g the gradients (MC_LIST_GRADS) times *coef:
 *     m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
 *     p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * and the model's copy, if the handle has one, is p rounded to its type.
 *   coef    device, one float (such as mc_grad_norm's out + 1), or NULL for 1.  0: the update is left out, nothing is written.
 * Errors: MC_ERR_INVALID_ARG (null, lists not bound, step < 1, betas outside [0, 1), eps <= 0, lr or weight_decay
 * negative or not finite, eps 0 or infinite in binary32, the factors 1 - lr weight_decay or lr / (1 - beta1^step) infinite there).
 */
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;             /* 1 for the first update */
} mc_adamw_config;
int mc_adamw(mc_step *h, const mc_adamw_config *cfg, const float *coef, void *stream);

/* ---- rows of logits ------------------------------------------------------------------------------------------- */
typedef struct mc_loss mc_loss;

/* Scratch for the calls below on the current HIP device (2 MB). */
int mc_loss_create(mc_loss **out);
int mc_loss_destroy(mc_loss *h);

/* Rows of logits, one per token: row r starts at logits + r * stride elements.  Entries of minus infinity have
 * probability 0 (places of a padded vocabulary, tokens that may not be chosen). */
typedef struct {
    const void *logits;       /* device                                                        */
    const int64_t *labels;    /* device, rows entries                                          */
    int64_t rows, vocab, stride;
    int32_t dtype;            /* mc_dtype of the logits                                        */
    float temperature;        /* > 0: the logits are divided by it                              */
} mc_logits;

/*
 * logp[r] = x_a - log(sum_j exp(x_j)), x the row's logits / temperature, a its label.
 * A row whose label lies outside [0, vocab) is not read; its logp is 0.
 *   logp   device, rows floats
 * Errors: MC_ERR_INVALID_ARG (null, negative sizes, vocab < 1, stride < vocab, unknown type, misaligned pointers, temperature,
 * logp over labels or logits), MC_ERR_RANGE (vocab of 2^31 - 2^16 or more, rows of 2^31 or more).
 */
int mc_token_logp(mc_loss *h, const mc_logits *x, float *logp, void *stream);

/*
 * Clipped policy loss with a KL term, over the rows that take part: those whose weight is not 0 and whose label lies in
 * [0, vocab).  With l the row's log-probability of its label as above, rho = exp(l - old_logp), A its advantage:
 *     policy = max(-A rho, -A clamp(rho, 1 - clip_low, 1 + clip_high))
 *     kl     = exp(ref_logp - l) - (ref_logp - l) - 1                    (0 without ref_logp)
 *     loss   = sum over the rows of weight * (policy + kl_coef kl)
 * Weights stand for masks and for how the loss is averaged (1 / tokens, or 1 / (sequences * tokens of the sequence)).
 * Gradient: dlogits = grad_scale * d loss / d logits, 0 in rows that take no part (their logits are not read).
 */
typedef struct {
    const float *old_logp;    /* device, rows                                                  */
    const float *advantages;  /* device, rows                                                  */
    const float *weights;     /* device, rows; NULL: all 1                                     */
    const float *ref_logp;    /* device, rows; NULL: no KL term                                */
    float clip_low, clip_high, kl_coef, grad_scale;
    float *sums;              /* device, 8 words: the sums over the rows that take part of weight * (policy + kl_coef kl),
                                 weight * policy, weight * kl, weight where the clamp decides, weight; then two int32: rows
                                 that take part, rows with a weight but no valid label; then 0  */
    float *logp;              /* device, rows, 0 where a row takes no part; may be NULL           */
    void *dlogits;            /* device, the logits' type; may be NULL (no gradient) or the logits themselves, of the same stride, but may
                                 not overlap them otherwise (columns or rows between theirs are no overlap)   */
    int64_t dlogits_stride;
} mc_policy;
/* Errors: as mc_token_logp, and MC_ERR_INVALID_ARG for null old_logp, advantages or sums, clip_low outside [0, 1], clip_high
 * or kl_coef negative, anything not finite, logp or dlogits over anything else, sums over either (or, with more than 2^17 rows, over
 * what is read). */
int mc_policy_loss(mc_loss *h, const mc_logits *x, const mc_policy *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MERGECOMP_STEP_H */
