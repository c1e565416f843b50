/*
 * cliffconv_ff.h -- C ABI of the residual feed-forward operators of
 * libcliffconv.so (MI355X, gfx950): what a network of Clifford linear layers
 * (cliffconv.h) has between them -- layer norm, dense layers with bias,
 * activation, dropout and residual in their epilogue, dropout by itself --
 * and their gradients.
 *
 * Tensors are matrices of rows: tokens, or the flattened multivectors
 * (C * N_B features) that clifford_linear reads and writes as [B, C, N_B].
 *
 * Common conventions (beside those of cliffconv.h on device pointers,
 * streams, threads and errors)
 *  - All tensors of a call have the one type `dtype`; statistics are fp32.
 *    Products are summed, and norms, activations and gradients computed, in
 *    fp32; each output is rounded to its type once, where not said otherwise.
 *  - A matrix is row-major with a row stride (leading dimension, in elements)
 *    of at least its width; the elements between rows are not touched.
 *    Vectors are contiguous.  Pointers are aligned to their element; 16-byte
 *    aligned rows are faster (base and row stride).
 *  - Sizes: widths are 1 to 2^31 - 1, row counts 0 to 2^31 - 1, and a matrix
 *    spans fewer than 2^40 elements (CLIFF_ESHAPE).  Without rows the matrices
 *    that have none may be NULL, and sums over rows are zero.
 *  - An output must not overlap an input, another output or the workspace
 *    (CLIFF_EOVERLAP), except where it may be the same matrix (same pointer
 *    and row stride).  Matrices that share a row stride and no column, such
 *    as two column ranges of one buffer, do not overlap.
 *  - Workspace: device memory of the caller, 16-byte aligned, at least as
 *    large as the operator's _workspace function says (0: NULL will do), else
 *    CLIFF_ESCRATCH.  Its contents are unspecified before and after; calls
 *    that may run at the same time need one each.
 *  - Results are the same bits from call to call: no sum depends on the order
 *    in which workgroups finish.
 *
 * Dropout: element (r, c) of a matrix (its row and column, whatever the
 * strides) is dropped where word c mod 4 of Philox4x32-7 (Salmon, Moraes,
 * Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) with the key
 * rng[0] and the counter (c div 4, r mod 2^32, r div 2^32, rng[1] mod 2^32) is
 * below round(p 2^32), and scaled by 1 / (1 - p) otherwise.  Dropped elements
 * are zero whatever their value, infinities and NaN among them.  The mask is
 * never stored: a gradient forms it again from the same p and rng.
 */
#ifndef CLIFFCONV_FF_H
#define CLIFFCONV_FF_H

#include <stdint.h>

#include "cliffconv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CLIFF_F32 = 0, CLIFF_BF16 = 1, CLIFF_F16 = 2 } cliff_dtype;

/* Pointwise activations f of a dense layer.  f(NaN) and f'(NaN) are NaN. */
typedef enum {
    CLIFF_ACT_NONE = 0,
    CLIFF_ACT_RELU = 1, /* max(v, 0); slope 0 at 0 */
    CLIFF_ACT_GELU = 2, /* v Phi(v), Phi the normal distribution function */
    CLIFF_ACT_SILU = 3  /* v / (1 + exp(-v)) */
} cliff_pointwise;

/*
 * Dropout of a matrix.  NULL or p = 0: none.
 *   p    probability, 0 <= p <= 1
 *   rng  device int64[2], 8-byte aligned: the generator's key (64 bits) and
 *        the step's number; read when the kernels run, so that a captured
 *        graph draws new masks once they are changed
 */
typedef struct {
    double p;
    const int64_t* rng;
} cliff_dropout_desc;

/*
 * Dense layer:
 *
 *   pre = x w + bias,   y = residual + dropout(f(pre))
 *
 *   x         [M, K], row stride ldx
 *   w         w_out_in = 0: [K, N] with row stride ldw (the order of
 *             clifford_linear's weight); 1: [N, K]
 *   bias      [N], or NULL for zero
 *   act       cliff_pointwise
 *   residual  [M, N], or NULL for zero; may be y
 *   pre       [M, N], written for the gradient, or NULL
 *   y         [M, N]
 * fp32 products are formed on the bf16 matrix cores from operands split into
 * three bf16 parts, as in cliffconv.h ("Precision").
 */
int64_t cliffconv_dense_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status cliffconv_dense(int dtype, int64_t M, int64_t K, int64_t N, const void* x,
                             int64_t ldx, const void* w, int64_t ldw, int w_out_in,
                             const void* bias, int act, const cliff_dropout_desc* drop,
                             const void* residual, int64_t ldr, void* pre, int64_t ldp, void* y,
                             int64_t ldy, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Gradient of the dense layer (the residual's is dy itself):
 *
 *   g = dropout(dy) f'(pre),   dx = g w^T,   dw = x^T g,   dbias = sum over rows of g
 *
 *   dy        [M, N]
 *   x, w      as in the forward call
 *   pre       [M, N] as the forward call wrote it; NULL where act is NONE
 *   dx        [M, K], or NULL: not wanted
 *   dw        in the order of w with row stride lddw, or NULL
 *   dbias     [N], or NULL
 * With GELU and SiLU, 16-bit types round g once before the two products (dbias
 * sums it unrounded): at most 2^-8 of each element in bf16, 2^-11 in fp16.  The
 * dropout's 1 / (1 - p) multiplies the sums, and a slope of 0 or 1 rounds nothing.
 */
int64_t cliffconv_dense_backward_workspace(int dtype, int64_t M, int64_t K, int64_t N);
cliff_status cliffconv_dense_backward(int dtype, int64_t M, int64_t K, int64_t N, const void* dy,
                                      int64_t lddy, const void* x, int64_t ldx, const void* w,
                                      int64_t ldw, int w_out_in, const void* pre, int64_t ldp,
                                      int act, const cliff_dropout_desc* drop, void* dx,
                                      int64_t lddx, void* dw, int64_t lddw, void* dbias,
                                      void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Layer norm over the d columns of each row:
 *
 *   mean = sum x / d,   rstd = 1 / sqrt(sum (x - mean)^2 / d + eps),
 *   y = (x - mean) rstd weight + bias
 *
 *   x, y       [rows, d]; y may be x
 *   weight     [d], or NULL for one
 *   bias       [d], or NULL for zero
 *   eps        >= 0
 *   mean, rstd fp32 [rows], written for the gradient, or NULL
 */
cliff_status cliffconv_layer_norm(int dtype, int64_t rows, int64_t d, const void* x, int64_t ldx,
                                  const void* weight, const void* bias, double eps, void* y,
                                  int64_t ldy, float* mean, float* rstd, void* stream);

/*
 * Gradient of the layer norm, with h = (x - mean) rstd and q = dy weight:
 *
 *   dx = rstd (q - mean(q) - h mean(q h)) + dresidual
 *   dweight = sum over rows of dy h,   dbias = sum over rows of dy
 *
 *   dy, x      [rows, d]
 *   mean, rstd fp32 [rows], as the forward call wrote them
 *   weight     [d], or NULL for one
 *   dresidual  [rows, d]: the gradient that the row gets past the norm, added
 *              before the rounding; NULL for zero; may be dx
 *   dx         [rows, d]; may be dy
 *   dweight, dbias  [d], each or NULL: not wanted
 */
int64_t cliffconv_layer_norm_backward_workspace(int dtype, int64_t rows, int64_t d);
cliff_status cliffconv_layer_norm_backward(int dtype, int64_t rows, int64_t d, const void* dy,
                                           int64_t lddy, const void* x, int64_t ldx,
                                           const float* mean, const float* rstd,
                                           const void* weight, const void* dresidual, int64_t ldr,
                                           void* dx, int64_t lddx, void* dweight, void* dbias,
                                           void* workspace, int64_t workspace_bytes,
                                           void* stream);

/*
 * Dropout, and its gradient (the same call on the gradient):
 *
 *   y = residual + dropout(x)
 *
 *   x, y      [rows, d]; y may be x or residual
 *   drop      not NULL
 *   residual  [rows, d], or NULL for zero
 */
cliff_status cliffconv_dropout(int dtype, int64_t rows, int64_t d, const void* x, int64_t ldx,
                               const cliff_dropout_desc* drop, const void* residual, int64_t ldr,
                               void* y, int64_t ldy, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CLIFFCONV_FF_H */
