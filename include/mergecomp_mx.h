/*
 * mergecomp_mx.h -- C ABI of a training step in few bits, in the same library as mergecomp.h and mergecomp_step.h.
 *
 *     mc_adamw8        mc_adamw with the moments held in 8 bits, over a model's list of tensors
 *     mc_mx_quantize   a matrix in microscaled 4-bit floating point, along rows and along columns
 *     mc_mx_matmul     the product of two such matrices
 *
 * Conventions: those of mergecomp_step.h.  A handle belongs to the device that was current when it was made, calls only enqueue kernels
 * on the caller's stream, allocate nothing and never synchronise, and all calls on one handle are issued in stream order, since they
 * share its scratch (calls captured into graphs too: graphs that hold calls on one handle are not replayed at the same time).  A captured
 * call keeps the numbers that it was made with (an update's step and rate too) and goes by the lists that are bound when it is replayed: the handle, what is
 * bound and the matrices have to be there until the last replay.  The same call gives the same bits.  What a call writes may not lie over anything else that it
 * writes or reads.
 */
#ifndef MERGECOMP_MX_H
#define MERGECOMP_MX_H

#include "mergecomp_step.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- AdamW with moments in 8 bits ------------------------------------------------------------------------------ */
/*
 * A moment is held in blocks of 128 consecutive elements of a tensor (the last one of a tensor may be shorter): a byte per element, an
 * 8-bit float c of four exponent and three mantissa bits (largest 448, least 2^-9, 0x7F and 0xFF not a number), and a binary32 scale s per
 * block.  The first moment is c s, the second (c s)^2: of it the root is held, which takes half the range of exponents.
 * After an update s is a block's largest magnitude / 448 and c = x / s rounded to nearest even, except that a root above 0 is never
 * rounded to 0, since updates are divided by it.  A block whose largest magnitude is below 2^-100 is held as zeros.  Infinities and NaN
 * leave the scale alone and are held as NaN, each in its own place, also where the rest of the block is held as zeros; the root of a square beyond
 * binary32 is one of them, though its gradient is finite.  Zero bytes and scales are moments of 0, which training begins with.
 * What rounding takes away is not kept.  An update that changes an element's ratio to the largest of its block by less than half a step of its
 * code (1/32 to 1/16 of it) leaves the code as it was, and such changes never add up; that largest itself is followed in 32 bits.  The first moment
 * falls by 1 - beta1 of itself in an update, more than that at 0.9.  A root falls by no more than 1 - sqrt(beta2): 2.5 percent at 0.95, 0.05
 * at 0.999.  Up to a beta2 of 0.98 the gradients' own variation, and the block's largest with it, moves codes often enough: after half of a block's normal
 * gradients became four times smaller their roots were within -12 and +13 percent (0.95; 5th to 95th percentile) and -15 and +29 (0.98) of the
 * true ones.  From 0.99 on roots do not come down: 2000 updates later they were 3 times the true ones (the median; 5000 later at 0.999 3.3), and
 * updates that much too small; where gradients end altogether a root can stay for good.  Gradients that grow are followed.  With such a beta2
 * take mc_adamw, whose moments have 32 bits, wherever gradients become smaller for long.
 */
typedef struct mc_step8 mc_step8;

typedef enum {
    MC_LIST8_GRADS = 0,            /* grad_dtype                                        */
    MC_LIST8_PARAMS = 1,           /* fp32 weights                                      */
    MC_LIST8_MODEL = 2,            /* model_dtype, as mc_list's                         */
    MC_LIST8_EXP_AVG = 3,          /* bytes, numel                                      */
    MC_LIST8_EXP_AVG_SQ = 4,       /* bytes, numel                                      */
    MC_LIST8_EXP_AVG_SCALE = 5,    /* fp32, ceil(numel / 128)                           */
    MC_LIST8_EXP_AVG_SQ_SCALE = 6, /* fp32, ceil(numel / 128)                           */
    MC_LISTS8 = 7
} mc_list8;

/* Arguments, limits and errors as mc_step_create; device memory: 16 bytes per 2048 elements of a tensor, 56 per tensor. */
int mc_step8_create(mc_step8 **out, const int64_t *numel, int32_t n_tensors, int32_t grad_dtype, int32_t model_dtype,
                    const uint8_t *no_decay);
int mc_step8_destroy(mc_step8 *h);
/* As mc_step_bind. */
int mc_step8_bind(mc_step8 *h, int32_t list, const void *const *ptrs, void *stream);
/* As mc_adamw: the same formulas in binary32 on the values that are held, weights from the new moments before they are rounded.
 * (A second moment below 2^-126 may count as 0, and what the first is divided by is at least 2^-126.)
 * coef: what mc_grad_norm leaves in out + 1, or NULL for 1; 0: nothing is written. */
int mc_adamw8(mc_step8 *h, const mc_adamw_config *cfg, const float *coef, void *stream);

/* ---- matrices in microscaled 4-bit floating point --------------------------------------------------------------- */
/*
 * rows x cols values in blocks of 32 consecutive ones of a row: an element is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7; + 8:
 * negative), times 2^(e - 127), e a byte per block.  e = 255: all of the block's values are NaN.
 *
 * Layout.  A row is padded to a multiple of 128 columns: steps = ceil(cols / 128).  In the padding codes are 0 and scales not 255.
 *   codes   tiles of 16 rows by 128 columns, 1024 bytes each, the tiles of 16 rows one behind the other along the columns:
 *           the 32 codes from column 128 s + 32 g of row r begin at byte  (((r / 16) * steps + s) * 64 + g * 16 + r % 16) * 16,
 *           two to a byte, the first one in the low four bits.
 *   scales  tiles of 64 rows by 128 columns, 256 bytes each:
 *           the one of that block is at byte  (((r / 64) * steps + s) * 64 + g * 16 + r % 16) * 4 + r / 16 % 4.
 * A wavefront's operand of a matrix instruction is one tile's 1024 bytes, and the scales of four such tiles a word per lane.
 * Rows that fill up the last tile are neither written nor do they reach a result.
 */
typedef struct {
    void *codes;              /* device, mc_mx_code_bytes, on a multiple of 16 bytes           */
    void *scales;             /* device, mc_mx_scale_bytes, on a multiple of 4 bytes           */
    int64_t rows, cols;       /* rows >= 0, cols >= 1, below 2^31 - 2^16                       */
} mc_mx_matrix;

/* Bytes of a matrix's buffers: ceil(rows / 16) * steps * 1024 and ceil(rows / 64) * steps * 256; 0 where rows or cols are out of range. */
size_t mc_mx_code_bytes(int64_t rows, int64_t cols);
size_t mc_mx_scale_bytes(int64_t rows, int64_t cols);

typedef struct mc_mx mc_mx;
/* Scratch for the calls below on the current HIP device (about 64 MB: sums of products that several blocks share). */
int mc_mx_create(mc_mx **out);
int mc_mx_destroy(mc_mx *h);

/*
 * Quantises x, rows x cols values of `dtype`, row r from data + r * stride elements on.  Every block of 32 gets the least power of two
 * under which its largest magnitude is at most 7 (6 and a rounding; at least 2^-127), and its values are rounded to nearest even.  A block
 * that holds an infinity or a NaN gets e = 255.
 *   by_rows   rows x cols, blocks along the rows; may be NULL
 *   by_cols   cols x rows, blocks along the columns: the transposed matrix, for products that sum over rows; may be NULL
 *   values    dtype, values_stride: what by_rows stands for, rounded to the type (beyond its range: its largest finite number; blocks
 *             with e = 255: NaN); may be NULL, or x itself with its stride
 * All in one launch, in which x is read once.
 * Errors: MC_ERR_INVALID_ARG (null, all three results null, negative sizes, cols < 1, strides below cols, unknown type, misaligned
 * pointers, matrices of other sizes, overlaps), MC_ERR_RANGE (rows or cols of 2^31 - 2^16 or more).
 */
typedef struct {
    const void *data;         /* device                        */
    int64_t rows, cols, stride;
    int32_t dtype;            /* mc_dtype                      */
} mc_mx_source;
int mc_mx_quantize(mc_mx *h, const mc_mx_source *x, const mc_mx_matrix *by_rows, const mc_mx_matrix *by_cols, void *values,
                   int64_t values_stride, void *stream);

/*
 * out[i][j] = sum_k a[i][k] b[j][k]  (+ bias[j])  (+ out[i][j] as it was, with `accumulate`)
 * Products and scales are exact, sums binary32 (what is below 2^-126 may count as 0); the result is rounded once, to nearest even.
 *   a          m x k, such as activations            b   n x k, such as weights of n outputs
 *   out        dtype, row i from out + i * stride elements on
 *   bias       device, n floats; may be NULL
 * With W quantised by rows (y = x W^T) the backward pass takes W by columns (dx = dy W) and dy and x by columns (dW = dy^T x).
 * Errors: MC_ERR_INVALID_ARG (null, a's and b's columns differ, sizes, stride < n, unknown type, misaligned pointers, overlaps),
 * MC_ERR_RANGE (m, n or k of 2^31 - 2^16 or more).
 */
typedef struct {
    void *out;                /* device                        */
    int64_t stride;
    int32_t dtype;            /* mc_dtype                      */
    int32_t accumulate;
    const float *bias;
} mc_mx_result;
int mc_mx_matmul(mc_mx *h, const mc_mx_matrix *a, const mc_mx_matrix *b, const mc_mx_result *y, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MERGECOMP_MX_H */
