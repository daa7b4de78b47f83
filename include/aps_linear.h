/*
 * aps_linear.h -- C ABI of the linear layers, their 8-bit activation
 * checkpoints and their gradients (libaps.so, beside aps.h).
 *
 * The calls form the gradients that the calls of aps.h synchronise: a
 * layer's forward product, what is kept of it for the backward pass, and the
 * backward pass itself, whose weight gradients are written as fp32 wherever
 * the caller wants them, e.g. at a layer's offset in a worker's row of G.
 *
 * A layer with weights W[N][K] (out features, in features):
 *   forward      z = X W^T + b,  Y = act(z) + R      X[M][K], Y, R, z [M][N]
 *   backward     dZ = dY * act'(z)                   (aps_activation_grad, or in the
 *                                                     epilogue of the next layer's aps_linear_grad_input)
 *                dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
 * The backward pass reads z and X from 8-bit checkpoints.
 *
 * Types.  X, W, b, R, Y, dY, dZ and dX of a call are all of one type, dtype;
 * dW and db are fp32.  Sums are held in fp32 and a result is rounded once,
 * to nearest even, when it is stored.  Matrices are row-major with a row
 * stride in elements, at least the row's length; pointers are aligned to
 * their element.  Rows of whole 16-byte chunks (8 or 4 elements, 16 codes)
 * that start on them (pointer and stride) run fastest; no alignment or length
 * is refused, others are copied or read in place.
 * Sizes: M, N, K in [0, 2^22] with every matrix at most 2^22 blocks of
 * 32 x 128 (2^34 elements); row strides up to 2^31 - 1.  Arrays that a
 * call does not touch (a dimension is 0) may be NULL.
 *
 * Checkpoints.  A matrix [M][C] is kept as one code byte per element,
 * codes[M][ldc], in 1-5-2 (bias 15) or 1-4-3 (bias 7), and one int32 word for
 * each block of APS_CKPT_ROWS x APS_CKPT_COLS elements (the last ones
 * partial): ckpt_exp[ceil(M / 32)][ceil(C / 128)], contiguous.  For a block:
 *   lim  = (2 - 2^-m) * 2^127, for APS_DTYPE_F16 (2 - 2^-m) * 2^15: the
 *          largest format value, times a power of two, that the type holds;
 *          a finite magnitude above lim is taken as lim
 *   ft   = min(emax - ceil(log2 max), APS_CKPT_MAX_EXP), max being the largest
 *          finite magnitude in the block; 0 where that is 0
 *   code = R_fmt(x * 2^ft), as aps_quantize's; INF and NaN keep theirs
 *   word = ft & 0xFFFF, plus 1 << 16 if an element of the block is INF or NaN
 * and the element stands for code's value * 2^-ft.  An INF or NaN costs only
 * its own element.  The value is exact in bfloat16 and fp32, and in half for
 * a checkpoint of halves (otherwise it is rounded to the nearest half).
 * Calls that read a checkpoint need ft in [-126, 126].
 *
 * Activations: none, max(z, 0), z * Phi(z) with the normal distribution's
 * Phi (the exact GELU), z / (1 + exp(-z)); at +-INF their limits.  The
 * derivative of max(z, 0) at 0 is 0.  A NaN gives NaN.  Of a given z, fp32
 * results are within 2^-20 of the function relative to themselves (derivatives
 * to their two terms), 16-bit ones within 2^-14 before they are rounded, as
 * long as exp(-z^2 / 2) of GELU or exp(-|z|) of SiLU is a normal fp32 number.
 *
 * Streams, errors and status codes are those of aps.h: arguments are checked
 * on the host before anything is enqueued on `stream`, and the contents of
 * device arrays are not.  Nothing is allocated and every call is a fixed sequence of kernels, so calls
 * can be captured in a HIP graph.  Results do not depend on the launch's
 * timing: there are no floating-point atomics.  An output overlaps no input,
 * except that Y may be R, dX may be R and dZ may be dY (same pointer and
 * stride).
 */
#ifndef APS_LINEAR_H
#define APS_LINEAR_H

#include "aps.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { APS_DTYPE_F32 = 0, APS_DTYPE_BF16 = 1, APS_DTYPE_F16 = 2 };
enum { APS_ACT_NONE = 0, APS_ACT_RELU = 1, APS_ACT_GELU = 2, APS_ACT_SILU = 3 };
enum { APS_LINEAR_FORWARD = 0, APS_LINEAR_GRAD_INPUT = 1, APS_LINEAR_GRAD_WEIGHT = 2 };
enum { APS_LINEAR_ON_CHUNKS = 4, APS_LINEAR_NO_CKPT = 8, APS_LINEAR_OFF_CHUNKS = 16 }; /* aps_linear_workspace_bytes: added to op */
#define APS_CKPT_ROWS 32
#define APS_CKPT_COLS 128
#define APS_CKPT_MAX_EXP 96
#define APS_GRAD_ACCUMULATE 1u /* aps_linear_grad_weight: add to dW and db */

/*
 * Bytes of workspace that aps_linear (op APS_LINEAR_FORWARD),
 * aps_linear_grad_input or aps_linear_grad_weight needs for a layer with M
 * rows, N out and K in features: the partial sums of a contraction that is
 * split over the GPU, and copies of operands whose rows are no whole 16-byte
 * chunks.  They suffice for every such call, and a workspace that is given
 * holds at least as many.  0 where none needs any, and for arguments out of
 * range.  Host-only.  Flags can be added to op:
 *   APS_LINEAR_ON_CHUNKS   of operands whose rows start on 16-byte chunks, less
 *                          than 2^21 elements apart, or are no whole ones: 0
 *                          where their call uses none; it can then be made
 *                          with workspace NULL and 0 bytes
 *   APS_LINEAR_OFF_CHUNKS  of operands whose rows are whole chunks but do not all
 *                          start on them, or lie further apart: more, where it
 *                          pays to copy such an operand first.  With the bytes
 *                          alone that every call needs it is read in place, up
 *                          to eight times slower, its sums in another order
 *   APS_LINEAR_NO_CKPT     of aps_linear without codes
 */
uint64_t aps_linear_workspace_bytes(int32_t op, int32_t M, int32_t N, int32_t K, int32_t dtype);

/*
 * z = X W^T + b;  Y = act(z) + R, and optionally the checkpoint of z (taken
 * from its fp32 value).
 *   X [M][ldx], W [N][ldw], Y [M][ldy]
 *   bias       [N], or NULL
 *   R          [M][ldr], or NULL
 *   codes      uint8 [M][ldc] out with ckpt_exp out, or NULL (then ckpt_fmt is
 *              not read)
 *   workspace  at least aps_linear_workspace_bytes(APS_LINEAR_FORWARD, ...)
 *              bytes, 16-byte aligned; calls that share one must not overlap.
 *              NULL with 0 bytes where the call uses none
 * K = 0 gives z = b.
 */
int aps_linear(const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias,
               const void* R, int64_t ldr, void* Y, int64_t ldy, int32_t M, int32_t N, int32_t K,
               int32_t dtype, int32_t act, aps_format ckpt_fmt, uint8_t* codes, int64_t ldc,
               int32_t* ckpt_exp, void* workspace, uint64_t workspace_bytes, void* stream);

/*
 * dX = (dZ W) * act'(z) + R, z [M][K] being the pre-activation that made this
 * layer's input, from its checkpoint.
 *   dZ [M][lddz], W [N][ldw], dX [M][lddx]
 *   act        APS_ACT_NONE: no factor (fmt, codes and ckpt_exp are not read)
 *   R          [M][ldr], e.g. the gradient that bypasses the layer, or NULL
 */
int aps_linear_grad_input(const void* dZ, int64_t lddz, const void* W, int64_t ldw, const void* R,
                          int64_t ldr, int32_t act, aps_format fmt, const uint8_t* codes, int64_t ldc,
                          const int32_t* ckpt_exp, void* dX, int64_t lddx, int32_t M, int32_t N,
                          int32_t K, int32_t dtype, void* workspace, uint64_t workspace_bytes,
                          void* stream);

/*
 * dW = dZ^T X, db = column sums of dZ, X [M][K] from its checkpoint.
 *   dZ [M][lddz], dW fp32 [N][lddw], db fp32 [N] or NULL
 *   flags      0 or APS_GRAD_ACCUMULATE (dW += ..., db += ...)
 * M = 0 gives zeros (nothing is added).  K = 0 with db returns APS_ERR_SIZE.
 */
int aps_linear_grad_weight(const void* dZ, int64_t lddz, aps_format fmt, const uint8_t* codes,
                           int64_t ldc, const int32_t* ckpt_exp, float* dW, int64_t lddw, float* db,
                           int32_t M, int32_t N, int32_t K, int32_t dtype, uint32_t flags,
                           void* workspace, uint64_t workspace_bytes, void* stream);

/* dZ = dY * act'(z), z [M][C] from its checkpoint. */
int aps_activation_grad(const void* dY, int64_t lddy, int32_t act, aps_format fmt,
                        const uint8_t* codes, int64_t ldc, const int32_t* ckpt_exp, void* dZ,
                        int64_t lddz, int32_t M, int32_t C, int32_t dtype, void* stream);

/* The checkpoint of X [M][ldx], C columns. */
int aps_checkpoint_save(const void* X, int64_t ldx, int32_t M, int32_t C, int32_t dtype,
                        aps_format fmt, uint8_t* codes, int64_t ldc, int32_t* ckpt_exp,
                        void* stream);

/* X = act(the checkpoint's values), in dtype: the activations again. */
int aps_checkpoint_load(const uint8_t* codes, int64_t ldc, const int32_t* ckpt_exp, int32_t M,
                        int32_t C, aps_format fmt, int32_t act, void* X, int64_t ldx, int32_t dtype,
                        void* stream);

#ifdef __cplusplus
}
#endif
#endif /* APS_LINEAR_H */
