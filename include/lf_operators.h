/* lf_operators.h -- C ABI of the operators of residual blocks, for one MI355X (gfx950): the root-mean-square norm with
 * the residual's addition, the matrix product with bias, activation and residual in its epilogue, both with their
 * backward passes, and activations kept in 8 bits, which the norm and the product write and the backward passes read; the
 * layer norm, the product of operands in 8 bits with a scale for each block of 128, both with their backward passes, and the
 * distillation loss with its gradient.
 * In the same library as lf.h, with its status codes; no handles: every call names all that it reads and writes.
 *
 * Conventions (beyond those of lf.h)
 *   - A matrix is row-major, `ld` elements from one row to the next, ld >= columns: slices of columns or rows of a
 *     larger matrix are matrices too.  Storage types are fp32 and bf16 (`data` aligned to its element), and 8 bits,
 *     below.  The matrices of one call have one storage type; those that may be in 8 bits instead are named.  A row
 *     is at most 8 MiB.  Rows that start at multiples of 16 bytes are read with the widest loads.
 *   - Any number of columns from 1 and of rows from 0 on.  With no rows the gradients that are sums over rows are
 *     written as zeros and nothing else is touched.
 *   - Sums, norms and what lies between an operator's inputs and its outputs are fp32; an output is rounded once, to
 *     nearest even.  (One rounding in between: the backward pass of a bf16 product rounds dz to bf16, for
 *     the matrix instructions take both operands in one type.)  Sums are taken in an order that the shape alone
 *     decides: the same call gives the same bits.
 *   - hip_stream is a stream of the current device, where all buffers are.
 *   - Calls only enqueue kernels on hip_stream: no allocation, no synchronisation, no memory kept from one call to
 *     the next.  They may be recorded in a HIP graph from the first call on.  Buffers are the caller's and must live until
 *     the work has run.  `workspace` is scratch that any later call on the same stream may use again; 256-byte aligned.
 *   - An output must not overlap an input or another output, except where stated.
 *   - Calls may be made from several threads at once; lf_operator_error() is the calling thread's.
 *
 * 8 bits (LF_MATRIX_E4M3).  The 32 columns 32 g .. 32 g + 31 of a row (the row's last group may have fewer) share a scale:
 * with m the largest magnitude among their finite values, the power 2^e of the least integer e >= -117 with
 * m <= 448 * 2^e.  A value v is kept as the e4m3 number nearest to v / 2^e (ties to even; one that 2^e would carry beyond
 * the largest bf16 number as 240, the number below), an infinity as a NaN.  `data`: one byte per value, 16-byte aligned,
 * ld a multiple of 32, so whole groups lie in every row's memory; what a writer leaves in the codes past the last
 * column is zero, and readers do not look at them.  `scales`: one byte e + 127 per group, scale_ld bytes from row to row.  Code times
 * scale is a bf16 number, so a matrix in 8 bits is an exact operand of bf16 and of fp32 arithmetic.  Readers also take bytes that are
 * not written here: 255 stands for a NaN, and of bytes below 10, 0 among them, 2^(byte - 127) times a code may lie between
 * bf16 numbers, to which bf16 operations round it.  Gradients pass through: the gradient with respect to a matrix in 8 bits
 * is that with respect to its values.
 *
 * Blocks of 128 (LF_MATRIX_E4M3_128, LF_MATRIX_E4M3_TILES).  The same codes and scale bytes, found the same way, with one scale for the
 * 128 columns 128 g .. 128 g + 127 of a row, or for the 128 x 128 values of rows 128 h .. and columns 128 g .. (h the scales' row).
 * ld is a multiple of 128, `scales` 4-byte aligned and scale_ld a multiple of 4, so whole groups and whole fours of scales lie
 * in every row's memory; what lies past the last column and past the last scale is written (zeros; scales anything), and not looked at.
 * Products read these operands as they are, and what they contract over lies along the rows of both: a backward pass takes
 * transposed matrices.  Their results in bf16 and in 8 bits come from instructions that add each eight consecutive products of a sum
 * in 14 bits of the largest one (2e-5 of a sum of random signs), those in fp32 from sums that are fp32 throughout; for the latter
 * a code times a scale of bytes above 246 that is beyond the largest bf16 number is an infinity. */
#ifndef LF_OPERATORS_H
#define LF_OPERATORS_H

#include "lf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LF_MATRIX_F32 = 0,
    LF_MATRIX_BF16 = 1,
    LF_MATRIX_E4M3 = 2,
    LF_MATRIX_E4M3_128 = 3,
    LF_MATRIX_E4M3_TILES = 4,
    LF_MATRIX_INT_RANGE = 0x7fffffff
} lf_matrix_type;

typedef struct {
    void* data;               /* device pointer to element (0, 0) */
    long long ld;             /* elements from a row to the next */
    unsigned char* scales;    /* 8 bits: device pointer to the scale of row 0, group 0; else not looked at */
    long long scale_ld;       /* bytes from a row's scales to the next row's */
    lf_matrix_type type;
} lf_matrix;

typedef enum {
    LF_ACT_NONE = 0,          /* z */
    LF_ACT_SIGMOID = 1,       /* 1 / (1 + e^-z) */
    LF_ACT_RELU = 2,          /* max(z, 0); its slope at 0 is 0 */
    LF_ACT_SILU = 3,          /* z / (1 + e^-z) */
    LF_ACT_GELU = 4,          /* z Phi(z), Phi the normal distribution function */
    LF_ACT_INT_RANGE = 0x7fffffff
} lf_activation;

/* Keep x (fp32 or bf16) in 8 bits. */
lf_status lf_checkpoint_save(int rows, int cols, const lf_matrix* x, const lf_matrix* out, void* hip_stream);

/* The values of a matrix in 8 bits, in fp32 or bf16 (exact in either). */
lf_status lf_checkpoint_load(int rows, int cols, const lf_matrix* in, const lf_matrix* out, void* hip_stream);

/* Root-mean-square norm with the residual's addition:
 *     s = x + branch,   rstd = 1 / sqrt(mean over the columns of s^2 + eps),   y = s rstd gain.
 * branch may be NULL (s = x).  sum (may be NULL) receives s; y is formed from s before that rounding.  y: storage type or
 * 8 bits.  gain: [cols] fp32, NULL for ones.  rstd: [rows] fp32, may be NULL.  sum may be x or branch itself (same data and ld).
 * LF_EINVAL unless eps is finite and >= 0. */
lf_status lf_norm_forward(int rows, int cols, const lf_matrix* x, const lf_matrix* branch, const float* gain, float eps,
                          const lf_matrix* sum, const lf_matrix* y, float* rstd, void* hip_stream);

/* Its backward pass: from dy, the gradient of y, and dsum, the gradient that reaches s on other ways (NULL: none),
 *     h = s rstd,  t = dy gain,   dx = dsum + rstd (t - h mean over the columns of (t h)),   dgain = sum over rows of dy h.
 * dx is the gradient of x and of branch.  sum: s, in storage type or 8 bits; rstd: as the forward pass gave it.  dgain ([cols]
 * fp32, overwritten) may be NULL, then no workspace is needed.  dx may be dsum itself. */
size_t lf_norm_workspace_bytes(int rows, int cols);
lf_status lf_norm_backward(int rows, int cols, const lf_matrix* dy, const lf_matrix* sum, const float* gain,
                           const float* rstd, const lf_matrix* dsum, const lf_matrix* dx, float* dgain,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/* Matrix product with bias, activation and residual:
 *     z = x w^T + bias,   y = act(z) + residual.
 * x: rows x inputs, storage type or 8 bits.  w: outputs x inputs (row-major as lf.h's w^l).  bias: [outputs] fp32, may be
 * NULL.  residual (may be NULL): rows x outputs.  y: rows x outputs, storage type or 8 bits.  z (may be NULL): what the
 * backward pass needs of an activation, rows x outputs, storage type or 8 bits. */
size_t lf_linear_workspace_bytes(int rows, int outputs, int inputs, lf_dtype dt);
lf_status lf_linear_forward(int rows, int outputs, int inputs, const lf_matrix* x, const lf_matrix* w, const float* bias,
                            lf_activation act, const lf_matrix* residual, const lf_matrix* y, const lf_matrix* z,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its backward pass, from dy, the gradient of y (and of residual):
 *     dz = dy act'(z),   dx = dz w,   dw = dz^T x,   db = sum over rows of dz.
 * z and x: storage type or 8 bits; z is not looked at for LF_ACT_NONE.  dx (rows x inputs), dw (outputs x inputs; fp32 or the
 * storage type) and db ([outputs] fp32) are overwritten; each may be NULL.  x may be NULL if dw is, w if dx is. */
size_t lf_linear_backward_workspace_bytes(int rows, int outputs, int inputs, lf_dtype dt);
lf_status lf_linear_backward(int rows, int outputs, int inputs, const lf_matrix* dy, const lf_matrix* z,
                             lf_activation act, const lf_matrix* x, const lf_matrix* w, const lf_matrix* dx,
                             const lf_matrix* dw, float* db, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Layer norm with the residual's addition:
 *     s = x + branch,   mean over the columns of s,   rstd = 1 / sqrt(mean over the columns of (s - mean)^2 + eps),
 *     y = (s - mean) rstd gain + shift.
 * As lf_norm_forward; y: storage type, LF_MATRIX_E4M3 or LF_MATRIX_E4M3_128.  gain, shift: [cols] fp32, NULL for ones, zeros.  mean,
 * rstd: [rows] fp32, may be NULL. */
lf_status lf_layer_norm_forward(int rows, int cols, const lf_matrix* x, const lf_matrix* branch, const float* gain,
                                const float* shift, float eps, const lf_matrix* sum, const lf_matrix* y, float* mean,
                                float* rstd, void* hip_stream);

/* Its backward pass: from dy, the gradient of y, and dsum, the gradient that reaches s on other ways (NULL: none),
 *     h = (s - mean) rstd,  t = dy gain,   dx = dsum + rstd (t - mean of t - h mean of (t h)),
 *     dgain = sum over rows of dy h,   dshift = sum over rows of dy.
 * sum: s, in storage type or LF_MATRIX_E4M3; mean, rstd: as the forward pass gave them.  dgain, dshift ([cols] fp32, overwritten) may be
 * NULL; without both no workspace is needed.  dx may be dsum itself. */
size_t lf_layer_norm_workspace_bytes(int rows, int cols);
lf_status lf_layer_norm_backward(int rows, int cols, const lf_matrix* dy, const lf_matrix* sum, const float* gain,
                                 const float* mean, const float* rstd, const lf_matrix* dsum, const lf_matrix* dx,
                                 float* dgain, float* dshift, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Keep x (rows x cols, fp32 or bf16) in 8 bits with blocks of 128: as it lies (out), transposed (out_t, cols x rows), or both.
 * Of LF_MATRIX_E4M3_128 the groups lie along each one's own rows; of LF_MATRIX_E4M3_TILES out_t holds out's codes.  Both have one type. */
lf_status lf_block_save(int rows, int cols, const lf_matrix* x, const lf_matrix* out, const lf_matrix* out_t, void* hip_stream);

/* The values of a matrix in 8 bits with blocks of 128, in fp32 or bf16. */
lf_status lf_block_load(int rows, int cols, const lf_matrix* in, const lf_matrix* out, void* hip_stream);

/* Matrix product of operands in 8 bits with blocks of 128, with bias, activation and residual:
 *     z = x w^T + bias,   y = act(z) + residual.
 * x: rows x inputs, LF_MATRIX_E4M3_128, or fp32 or bf16 that the call keeps so first.  w: outputs x inputs, LF_MATRIX_E4M3_TILES or
 * LF_MATRIX_E4M3_128.  residual, y, z as in lf_linear_forward, in fp32 or bf16; y and z may be LF_MATRIX_E4M3_128.  x_t (may be
 * NULL): inputs x rows, LF_MATRIX_E4M3_128, receives x transposed for the backward pass; x has to be fp32 or bf16 then. */
size_t lf_block_linear_workspace_bytes(int rows, int outputs, int inputs);
lf_status lf_block_linear_forward(int rows, int outputs, int inputs, const lf_matrix* x, const lf_matrix* w, const float* bias,
                                  lf_activation act, const lf_matrix* residual, const lf_matrix* y, const lf_matrix* z,
                                  const lf_matrix* x_t, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Its backward pass, from dy, the gradient of y (and of residual), fp32 or bf16:
 *     dz = dy act'(z),   dx = dz w,   dw = dz^T x,   db = sum over rows of dz.
 * dz is kept in 8 bits for the products, with groups along its outputs for dx and along its rows for dw; db is summed before that.
 * z: dy's type or LF_MATRIX_E4M3_128; not looked at for LF_ACT_NONE.  x_t: inputs x rows, LF_MATRIX_E4M3_128.  w_t: inputs x outputs,
 * LF_MATRIX_E4M3_TILES or LF_MATRIX_E4M3_128.  dx (rows x inputs; dy's type), dw (outputs x inputs; fp32 or dy's type) and db
 * ([outputs] fp32) are overwritten; each may be NULL.  x_t may be NULL if dw is, w_t if dx is. */
size_t lf_block_linear_backward_workspace_bytes(int rows, int outputs, int inputs);
lf_status lf_block_linear_backward(int rows, int outputs, int inputs, const lf_matrix* dy, const lf_matrix* z,
                                   lf_activation act, const lf_matrix* x_t, const lf_matrix* w_t, const lf_matrix* dx,
                                   const lf_matrix* dw, float* db, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Distillation from a teacher's top logits, the loss of each row and its gradient in one pass:
 *     p = softmax(t / T) over the row's `top` entries,   q = softmax(z / T) over the classes,
 *     loss = weight T^2 (sum over the entries of p (log p - log q)),   dlogits = weight T (q - p).
 * logits: z, rows x classes.  top_logits: t, rows x top, fp32 or bf16, whatever z is.  top_classes: the entries' classes, a row every
 * top_classes_ld elements; one that is negative is no entry, a class that occurs twice counts twice, and one >= classes makes the
 * row's loss and gradient NaN.  T = temperature, 2^-20 to 2^20.  weight: [rows] fp32, NULL for ones; a row of weight 0, or
 * without an entry above minus infinity, is not looked at further: its loss and gradient are zeros.  loss: [rows] fp32, may be NULL.  dlogits:
 * z's type, may be NULL, may be logits itself.  top: 1 to 1024. */
lf_status lf_distil(int rows, int classes, int top, const lf_matrix* logits, const lf_matrix* top_logits,
                    const int* top_classes, long long top_classes_ld, float temperature, const float* weight, float* loss,
                    const lf_matrix* dlogits, void* hip_stream);

/* Description of the calling thread's last failed call of this header.  Never NULL. */
const char* lf_operator_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LF_OPERATORS_H */
