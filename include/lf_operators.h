/* lf_operators.h -- C ABI of the operators of residual blocks, for one MI355X (gfx950): the root-mean-square norm with
 * the residual's addition, the matrix product with bias, activation and residual in its epilogue, both with their
 * backward passes, and activations kept in 8 bits, which the norm and the product write and the backward passes read.
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
 * is that with respect to its values. */
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
    LF_MATRIX_INT_RANGE = 0x7fffffff
} lf_matrix_type;

typedef struct {
    void* data;               /* device pointer to element (0, 0) */
    long long ld;             /* elements from a row to the next */
    unsigned char* scales;    /* LF_MATRIX_E4M3: device pointer to the scale of row 0, group 0; else not looked at */
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

/* Description of the calling thread's last failed call of this header.  Never NULL. */
const char* lf_operator_error(void);

#ifdef __cplusplus
}
#endif
#endif /* LF_OPERATORS_H */
