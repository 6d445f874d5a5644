/*
 * Training in reduced precision next to the optimizer step of tula_ags.h: the global gradient norm
 * and clipping, AdamW on fp32 master weights, Muon, microscaled 4-bit matrices (MXFP4), 8-bit
 * floating-point ones, and layer norm.  Part of libtula_ags.
 *
 * Conventions are those of tula_ags.h: caller-owned device memory; calls are asynchronous on
 * `stream` (a cudaStream_t; NULL = the legacy default stream), allocate nothing, never synchronize
 * the host and can be captured into a CUDA graph (the plans' creation is the exception, see
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
 * depends on M, N and K only; the sum is rounded once.  (They cut their sums off, with every 64 columns: a sum of
 * one sign may lose K 2^-29 of itself.)  A row with a NaN scale gives NaN.
 * M, N, K >= 0 (K = 0 gives zeros).
 */
int tula_mx_matmul(const void *a_codes, const void *a_scales, const void *b_codes,
                   const void *b_scales, int64_t M, int64_t N, int64_t K, void *out, int out_type,
                   void *stream);

/*
 * The error word of the MXFP4 kernels on the current device, read after the work already enqueued on
 * `stream` (the call waits for that stream), then cleared: 0 when every bounded wait inside the
 * kernels completed; bit 0 set when one ran out, bit 1 when shared memory did not start where a
 * product's kernel needs it, and the results since the last read are then not valid.
 */
int tula_mx_error(void *stream, int *error_out);

/* Failure-detection check: launches, on `stream`, one warp that waits, with the kernels' bound, on a
 * barrier that nothing arrives on (about two seconds) and records it as they do: tula_mx_error then
 * reports bit 0.  The CUDA context stays usable. */
int tula_mx_check_wait_timeout(void *stream);

/* ---------------------------------------------------------------------------------------------
 * 8-bit floating-point matrices with a scale for each block of 128
 * ------------------------------------------------------------------------------------------ */

/* Codes: E4M3 (largest 448) and E5M2 (largest 57344). */
#define TULA_FP8_E4M3 0
#define TULA_FP8_E5M2 1

/*
 * A rows x cols matrix of 8-bit codes: blocks of 128 elements along a row (the last one of a row may
 * be shorter), or of 128 rows by 128 columns, share a scale 2^(s - 127), s an E8M0 byte (255: NaN).
 * With P = cols rounded up to a multiple of 128:
 *   codes   [rows][P] bytes; zero beyond the matrix
 *   scales  [ceil(rows / 128)][ceil(P / 512)] tiles of 512 bytes, each of 128 rows by 4 blocks of
 *           columns: byte (row % 32) * 16 + (row % 128) / 32 * 4 + block % 4; zero beyond the matrix.
 *           (A block of 128 rows has its scale in each of them: what reads the matrix need not know.)
 * Both 16-byte aligned.
 */
/* Bytes of a matrix; sizes as for tula_mx_size. */
int tula_fp8_size(int64_t rows, int64_t cols, size_t *code_bytes, size_t *scale_bytes);

/*
 * Quantises x, device [rows][stride] of `type` (stride >= cols, in elements), to `code`: the scale is
 * the least power of two (2^-127 at least) that brings the block's largest magnitude to the code's
 * largest value or below, elements are x / 2^(s - 127) to the nearest code, ties to the even one; the
 * division is exact.  A block with an infinity or NaN gets s = 255 and codes 0.
 *   square             blocks of 128 x 128 (1) or of 1 x 128 (0)
 *   codes, scales      x itself; both or neither
 *   codes_t, scales_t  its transpose (cols x rows), blocks along x's columns (square: the same blocks);
 *                      both or neither
 * One pair at least; with both, x is read once.  rows, cols >= 0 (0: nothing is done).
 */
int tula_fp8_quantize(const void *x, int type, int64_t rows, int64_t cols, int64_t stride, int code,
                      int square, void *codes, void *scales, void *codes_t, void *scales_t,
                      void *stream);

/* The values a matrix stands for, rounded to `type`, into out, device [rows][cols]. */
int tula_fp8_dequantize(const void *codes, const void *scales, int64_t rows, int64_t cols, int code,
                        void *out, int type, void *stream);

/*
 * out = A B^T, A an M x K and B an N x K matrix of 8-bit codes (each of its own kind of code); out
 * device [M][N] of `out_type`.  As tula_mx_matmul: products of codes and scales are exact and added in
 * fp32 by the tensor cores in an order that depends on M, N and K only; the sum is rounded once.  (Here sums are
 * cut off with every 32 columns: K 2^-28.)
 */
int tula_fp8_matmul(const void *a_codes, const void *a_scales, int a_code, const void *b_codes,
                    const void *b_scales, int b_code, int64_t M, int64_t N, int64_t K, void *out,
                    int out_type, void *stream);

/*
 * A layer's forward pass, y = x w^T, in one call: x (M x K, blocks of 1 x 128) and w (N x K, blocks of
 * 128 x 128) quantised to `code`, and their product in x's type into y, device [M][N].  What the
 * backward pass multiplies by is left in `kept`: with need_dw x^T (K x M, blocks along the rows of x),
 * then with need_dx w^T (K x N), each its scales and then its codes (sizes of tula_fp8_size).  temp
 * holds x and w quantised, laid out so, and may be used again by what is enqueued after.  Both
 * 16-byte aligned, NULL where they would be empty (TULA_ERR_WORKSPACE otherwise).
 */
typedef struct tula_fp8_operand {
    const void *data;  /* device; row r, column c at r * stride + c, or with transposed c * stride + r */
    int64_t stride;    /* in elements, at least the length of what is contiguous */
    int type;          /* TULA_TYPE_* */
    int transposed;
} tula_fp8_operand;
int tula_fp8_linear(const tula_fp8_operand *x, const tula_fp8_operand *w, int64_t M, int64_t N,
                    int64_t K, int code, int need_dx, int need_dw, void *kept, void *temp, void *y,
                    void *stream);

/*
 * Its backward pass: dy (M x N) quantised to grad_code along the dimension that each product sums over,
 * dx = dy w (need_dx) into dx, device [M][K], and dw = dy^T x (need_dw) into dw, device [N][K].  `code`,
 * `kept` and what is needed are the forward pass's; temp holds dy (need_dx), then dy^T (need_dw).
 */
int tula_fp8_linear_backward(const tula_fp8_operand *dy, int64_t M, int64_t N, int64_t K, int code,
                             int grad_code, const void *kept, void *temp, void *dx, int dx_type,
                             void *dw, int dw_type, int need_dx, int need_dw, void *stream);

/* The error word of the 8-bit products and its check, as tula_mx_error and tula_mx_check_wait_timeout. */
int tula_fp8_error(void *stream, int *error_out);
int tula_fp8_check_wait_timeout(void *stream);

/* ---------------------------------------------------------------------------------------------
 * Layer norm
 * ------------------------------------------------------------------------------------------ */

/*
 * y = (x - mean) r w + b for each row of x, device [rows][stride] of `type` (stride >= cols, in
 * elements), mean and var (the mean of (x - mean)^2) over its cols elements, r = 1 / sqrt(var + eps);
 * y device [rows][cols] of `type`.  weight and bias: device [cols] of param_type, or NULL (1 and 0).
 * stats: device fp32 [rows][2], mean and r for the backward pass, or NULL.  In fp32, rounded once (the
 * sum of x and those of x - mean and its square have to lie in its range); errors are of the size of x - mean, not
 * of x, but for the mean in stats, which is one fp32 number.  A row with an infinity or NaN gives NaN.  rows below
 * 2^40, cols up to 2^24, eps >= 0 (TULA_ERR_ARG).
 */
int tula_layer_norm(const void *x, int type, int64_t rows, int64_t cols, int64_t stride,
                    const void *weight, const void *bias, int param_type, float eps, void *y,
                    float *stats, void *stream);

/*
 * Its gradients.  With n = (x - mean) r and g = dy w:
 *   dx = r (g - mean(g) - n mean(g n)),  dweight = sum of dy n,  dbias = sum of dy  (over the rows)
 * dy device [rows][dy_stride], x and stats of the forward pass; dx device [rows][cols] of `type`,
 * dweight and dbias device [cols] of param_type; each of the three may be NULL.  The sums over the rows
 * are taken in fp32 in an order that depends on the sizes and the device, rounded once.  The
 * workspace, of tula_layer_norm_workspace_size bytes (16-byte aligned, any contents), is needed for
 * dweight and dbias and may be used again by what is enqueued after.
 */
int tula_layer_norm_workspace_size(int64_t rows, int64_t cols, size_t *bytes);
int tula_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t stride, int type,
                             int64_t rows, int64_t cols, const void *weight, int param_type,
                             const float *stats, void *dx, void *dweight, void *dbias,
                             void *workspace, size_t workspace_bytes, void *stream);

/* The error word of these kernels and its check, as tula_mx_error and tula_mx_check_wait_timeout. */
int tula_layer_norm_error(void *stream, int *error_out);
int tula_layer_norm_check_wait_timeout(void *stream);

/* ---------------------------------------------------------------------------------------------
 * Orthogonalised updates (Muon)
 * ------------------------------------------------------------------------------------------ */

/*
 * O(u): u / |u| (the Frobenius norm; a matrix of zeros stays) and then ns_steps of
 *   X <- a X + b A X + c A^2 X,  A = X X^T,  (a, b, c) = (3.4445, -4.7750, 2.0315)
 * which bring the singular values near 1 (to 0.7 to 1.2 in five steps) and leave the singular vectors.
 * Operands are held in fp16 and summed in fp32: X, A and B are rounded in each step.  Relative to its norm O is
 * then off by
 *   0.5 to 2e-3   where most singular values are within 20 of the largest one,
 *   up to 1e-2    where the smaller side is 2 to 7 (a few values, whose roundings do not average),
 *   more          the more of them lie far below the largest ones, whose roundings grow with the small ones: 3e-3 for
 *                 1, 1/2, 1/3, ..., 2e-2 for their squares, 2 to 5e-2 with four 1000 times the others;
 * but for narrow matrices always by about as much as rounding the matrix to bf16 moves O, or less (a seventh of it in
 * the last two).  A matrix with an infinity or NaN gives NaN.
 */

/*
 * O of each of `batch` matrices x, device [rows][stride] of `type`, batch_stride elements apart
 * (stride >= cols, batch_stride >= 0), into out, device [batch][rows][cols] of out_type, bf16 or fp16.
 * ns_steps in [0, 100], rows and cols up to 2^20 (TULA_ERR_ARG).  The workspace (256-byte aligned, any
 * contents; some 4 to 8 bytes an element, of tiles of 128 x 64, TULA_ERR_ARG beyond 256 GB) may be used again by what is
 * enqueued after; calls that share one must be ordered.  Sums depend on sizes and alignments only.
 */
int tula_orthogonalize_workspace_size(int64_t batch, int64_t rows, int64_t cols, size_t *bytes);
int tula_orthogonalize(const void *x, int type, int64_t batch, int64_t rows, int64_t cols,
                       int64_t stride, int64_t batch_stride, int ns_steps, void *out, int out_type,
                       void *workspace, size_t workspace_bytes, void *stream);

/* A list of matrices.  HOST arrays of n_matrices entries, read by tula_muon_plan_create only; what
 * they point to is device memory, contiguous [rows][cols], aligned to its element (matrices whose columns are a
 * multiple of eight, whose weights start at 32 bytes and whose other buffers start at 16 move eight at a time, and
 * the last product writes their weights). */
typedef struct tula_muon_matrices {
    int n_matrices;
    const int64_t *rows, *cols;        /* >= 0 (0: skipped), up to 2^20 */
    void *const *grad_ptrs;
    const int *grad_types;             /* TULA_TYPE_*; NULL: all fp32 */
    float *const *param_ptrs;          /* fp32 weights */
    float *const *momentum_ptrs;       /* fp32, zero before the first step */
    void *const *copy_ptrs;            /* copies of the weights for the model, or NULL */
    const int *copy_types;             /* TULA_TYPE_BF16 or TULA_TYPE_F16; NULL: all bf16 */
} tula_muon_matrices;

/* Bytes of device workspace a plan over these sizes needs (host only): some 4 to 8 an element, of tiles of
 * 128 x 64; a few for a list of matrices that an SM's shared memory holds (smaller sides up to 128).
 * TULA_ERR_ARG for sizes beyond the limits and for more than 256 GB. */
int tula_muon_workspace_size(const int64_t *rows, const int64_t *cols, int n_matrices, size_t *bytes);

/* A plan, as tula_train_plan_create's: the same contract, errors and lifetime.  A buffer of weights,
 * momentum or copies that shares memory with another of the list is TULA_ERR_ARG (gradients may with each other, and
 * lie within their own matrix's weights or copy, which then overwrite them). */
typedef struct tula_muon_plan tula_muon_plan;
int tula_muon_plan_create(const tula_muon_matrices *matrices, void *workspace, size_t workspace_bytes,
                          void *stream, tula_muon_plan **plan_out);
int tula_muon_plan_destroy(tula_muon_plan *plan);

#define TULA_MUON_SCALE_RMS 0    /* 0.2 sqrt(max(rows, cols)): updates as large as AdamW's */
#define TULA_MUON_SCALE_ASPECT 1 /* sqrt(max(1, rows / cols)) */

typedef struct tula_muon_hparams {
    double lr, momentum, weight_decay;
    double grad_scale;    /* the loss scale: a factor the gradients hold (1: none) */
    int nesterov;         /* what is orthogonalised: d + momentum m (1) or m (0) */
    int ns_steps;         /* 0 to 100 */
    int scale;            /* TULA_MUON_SCALE_* */
    const float *record;  /* device fp32 [TULA_RECORD_LEN] as tula_grad_norm leaves it, or NULL: gradients
                             are clipped by its coefficient, and with a norm that is not finite the step
                             changes nothing */
} tula_muon_hparams;

/* lr 1e-3, momentum 0.95, no weight decay, grad_scale 1, nesterov, five steps, SCALE_RMS, no record. */
void tula_muon_default_hparams(tula_muon_hparams *hp);

/*
 * One step of Muon (Jordan et al., 2024: momentum orthogonalised by Newton-Schulz steps).  With c the
 * record's coefficient (1 without one) and s the shape's scale, for each matrix:
 *   d = g * (c / grad_scale),  m = momentum m + d,  u = d + momentum m or m
 *   w = w (1 - lr weight_decay) - lr s O(u)
 * in fp32 but for O, and the copies w rounded to their type.  Gradients are read only.  0 <= momentum < 1;
 * TULA_ERR_ARG for other values, for NaN, for grad_scale outside [2^-100, 2^100], for lr or weight_decay
 * outside [0, 1e30], for an unknown scale, and when the current device is not the plan's.
 */
int tula_muon_step(tula_muon_plan *plan, const tula_muon_hparams *hp, void *stream);

/* The error word of these products and its check, as tula_mx_error and tula_mx_check_wait_timeout. */
int tula_muon_error(void *stream, int *error_out);
int tula_muon_check_wait_timeout(void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TULA_TRAIN_H */
