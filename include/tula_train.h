/*
 * Training in reduced precision next to the optimizer step of tula_ags.h: the global gradient norm
 * and clipping, AdamW on fp32 master weights, and microscaled 4-bit matrices (MXFP4).  Part of
 * libtula_ags.
 *
 * Conventions are those of tula_ags.h: caller-owned device memory; calls are asynchronous on
 * `stream` (a cudaStream_t; NULL = the legacy default stream), allocate nothing, never synchronize
 * the host and can be captured into a CUDA graph (tula_train_plan_create is the exception, see
 * there); the return value is TULA_OK or a TULA_ERR_* code, and argument errors are detected on
 * the host before anything is enqueued; results are bitwise reproducible run to run.
 */
#ifndef TULA_TRAIN_H
#define TULA_TRAIN_H

#include "tula_ags.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define TULA_TYPE_F32 0
#define TULA_TYPE_BF16 1
#define TULA_TYPE_F16 2

/* ---------------------------------------------------------------------------------------------
 * The global gradient norm, clipping and AdamW over a list of tensors
 * ------------------------------------------------------------------------------------------ */

/* A list of tensors.  The arrays are HOST arrays of n_tensors entries, read by
 * tula_train_plan_create only; what they point to is device memory, aligned to its element.
 * Tensors whose buffers start alike within eight elements (all at a boundary of eight, or views at
 * one element offset into flat buffers that start at such boundaries) move eight elements at a
 * time, others one by one. */
typedef struct tula_train_tensors {
    int n_tensors;
    const int64_t *numels;             /* >= 0 (0 = skipped) */
    void *const *grad_ptrs;            /* gradients */
    const int *grad_types;             /* TULA_TYPE_*; NULL: all fp32 */
    float *const *param_ptrs;          /* fp32 weights and moments: all three, or all NULL for a */
    float *const *exp_avg_ptrs;        /* plan that takes norms and clips only */
    float *const *exp_avg_sq_ptrs;
    void *const *copy_ptrs;            /* copies of the weights for the model, or NULL */
    const int *copy_types;             /* TULA_TYPE_BF16 or TULA_TYPE_F16; NULL: all bf16 */
} tula_train_tensors;

/* Bytes of device workspace a plan over these sizes needs (host only): 64 to 72 per tile of 2048
 * elements (up to about 2.5 M elements in all) or 4096, and for what is left of each tensor. */
int tula_train_workspace_size(const int64_t *numels, int n_tensors, size_t *bytes);

/*
 * A plan: the list with its pointers and tiles laid out in the workspace (256-byte aligned, any
 * contents).  The copy to the device is made on `stream`, which the call waits for, so it cannot
 * be captured; everything after it can.  The tensors and the workspace must live as long as the
 * plan; calls that share a plan must be ordered.  Binds the plan to the current device.
 * Errors: TULA_ERR_ARG (NULL, misaligned or negative, an unknown type, 2^31 tiles or more),
 * TULA_ERR_WORKSPACE, TULA_ERR_CUDA, TULA_ERR_NO_MEMORY; *plan_out is NULL on error.
 * tula_train_plan_destroy frees host memory only; NULL is a no-op.
 */
typedef struct tula_train_plan tula_train_plan;
int tula_train_plan_create(const tula_train_tensors *tensors, void *workspace,
                           size_t workspace_bytes, void *stream, tula_train_plan **plan_out);
int tula_train_plan_destroy(tula_train_plan *plan);

/* What a norm leaves in a record, device fp32 [TULA_RECORD_LEN]. */
#define TULA_RECORD_NORM 0   /* |G| over all gradients, each divided by grad_scale (inf here above fp32's
                                range; what follows from it then is computed in fp64, as it is wherever
                                fp32 would leave its normal range on the way) */
#define TULA_RECORD_COEF 1   /* min(1, max_norm / (|G| + 1e-6)); 1 without a max_norm */
#define TULA_RECORD_FINITE 2 /* 1 if |G| is finite, else 0 */
#define TULA_RECORD_LEN 4    /* the last word is left as it is */

/*
 * |G| = sqrt(sum over all tensors and elements of g^2) / grad_scale, into the record.  Gradients
 * are read only.  Squares are summed in fp32 within 32 elements of a thread and its warp (with an
 * exact power of two taken out where they would overflow or underflow, so that the norm holds over
 * the whole range of the types) and in fp64 beyond, in an order that depends on the sizes and
 * alignments only.  An infinity in the gradients gives inf, a NaN gives NaN.  grad_scale lies in
 * [2^-100, 2^100].
 */
int tula_grad_norm(tula_train_plan *plan, float grad_scale, float max_norm, float *record,
                   void *stream);

/*
 * The norm as above (grad_scale 1), then g = coef * g for every gradient, in fp32, rounded once to
 * its type.  max_norm > 0.  With coef = 1 the gradients are left as they are; an infinite norm has
 * coef 0, whatever max_norm, and a NaN norm the coef NaN.
 */
int tula_grad_clip(tula_train_plan *plan, float max_norm, float *record, void *stream);

typedef struct tula_adamw_hparams {
    double lr, beta1, beta2, eps, weight_decay;
    double grad_scale;  /* the loss scale: a factor the gradients hold (1: none) */
    double max_norm;    /* > 0: clip by the global norm; 0: no clipping */
    int skip_nonfinite; /* 1: a step whose |G| is not finite changes nothing but steps[1] */
    float *record;      /* device fp32 [TULA_RECORD_LEN]; NULL only with max_norm 0 and no skip */
    int64_t *steps;     /* device [2]: steps taken, steps left out */
} tula_adamw_hparams;

/* lr 1e-3, betas 0.9 and 0.999, eps 1e-8, weight_decay 0.01, grad_scale 1, no clipping, no skip. */
void tula_adamw_default_hparams(tula_adamw_hparams *hp);

/*
 * One AdamW step (Loshchilov and Hutter, "Decoupled weight decay regularization").  With t the
 * steps taken before and including this one, c the clipping coefficient, per element in fp32:
 *   d = g * (c / grad_scale)
 *   m = beta1 m + (1 - beta1) d
 *   v = beta2 v + (1 - beta2) d^2
 *   w = w (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * and the copies w rounded to their type.  Gradients are read only (clipping does not write them).
 * The norm is taken, and the record written, only with a max_norm or skip_nonfinite.
 * 0 <= beta < 1; TULA_ERR_ARG for other values, for NaN, for grad_scale outside [2^-100, 2^100], lr, eps,
 * weight_decay or max_norm < 0, and for a plan without weights.
 */
int tula_adamw_step(tula_train_plan *plan, const tula_adamw_hparams *hp, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Microscaled 4-bit matrices (MXFP4, OCP Microscaling Formats 1.0)
 * ------------------------------------------------------------------------------------------ */

/*
 * A rows x cols matrix in MXFP4: blocks of 32 elements along a row (the last one of a row may be
 * shorter) share a scale 2^(s - 127), s an E8M0 byte (255: NaN); an element is an E2M1 code, the
 * sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  With P = cols rounded up to a multiple of 128:
 *   codes   [rows][P / 2] bytes, two codes a byte, the even column in the low half; zero beyond
 *           the matrix
 *   scales  [ceil(rows / 128)][P / 128] tiles of 512 bytes, each of 128 rows by 4 blocks: byte
 *           (row % 32) * 16 + (row % 128) / 32 * 4 + block % 4, the order in which the tensor
 *           cores take them; zero beyond the matrix
 * Both 16-byte aligned.
 */
/* Bytes of a matrix; rows and cols below 2^31 - 1023, at most 2^31 tiles (TULA_ERR_ARG). */
int tula_mx_size(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes);

/*
 * Quantises x, device [rows][stride] of `type` (stride >= cols, in elements): s = max(0, e - 2)
 * with e the biased exponent of the block's largest magnitude (so that it lands in [4, 8)), and
 * elements x / 2^(s - 127) to the nearest code, ties to the even one, magnitudes above 6 to 6; the
 * division is exact.  A block with an infinity or NaN gets s = 255 and codes 0.
 *   codes, scales      x itself, blocks along its rows; both or neither
 *   codes_t, scales_t  its transpose (cols x rows), blocks along x's columns; both or neither
 * One pair at least; with both, x is read once.  rows, cols >= 0 (0: nothing is done).
 */
int tula_mx_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride,
                     void *codes, void *scales, void *codes_t, void *scales_t, void *stream);

/* The values a matrix stands for, rounded to `type`, into out, device [rows][cols]. */
int tula_mx_dequantize(const void *codes, const void *scales, int64_t rows, int64_t cols,
                       void *out, int type, void *stream);

/*
 * out = A B^T, A an M x K and B an N x K matrix in MXFP4; out device [M][N] of `out_type`.
 * Products of codes and scales are exact and added in fp32 by the tensor cores in an order that
 * depends on M, N and K only; the sum is rounded once.  A row with a NaN scale gives NaN.
 * M, N, K >= 0 (K = 0 gives zeros).
 */
int tula_mx_matmul(const void *a_codes, const void *a_scales, const void *b_codes,
                   const void *b_scales, int64_t M, int64_t N, int64_t K, void *out, int out_type,
                   void *stream);

/*
 * The error word of these kernels on the current device, read after the work already enqueued on
 * `stream` (the call waits for that stream), then cleared: 0 when every bounded wait inside the
 * kernels completed; bit 0 set when one ran out, bit 1 when shared memory did not start where a
 * product's kernel needs it, and the results since the last read are then not valid.
 */
int tula_mx_error(void *stream, int *error_out);

/* Failure-detection check: launches, on `stream`, one warp that waits, with the kernels' bound, on a
 * barrier that nothing arrives on (about two seconds) and records it as they do: tula_mx_error then
 * reports bit 0.  The CUDA context stays usable. */
int tula_mx_check_wait_timeout(void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TULA_TRAIN_H */
