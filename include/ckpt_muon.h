/*
 * ckpt_muon.h -- C ABI of the optimizer step that orthogonalises a matrix's
 * update, and of the orthogonalisation alone.
 *
 * It stands beside ckpt_adamw (ckpt_ops.h): matrices inside a model take this
 * step, its tables and vectors AdamW's.  A matrix has one fragment less to
 * capture than with AdamW: parameter, fp32 master copy, one moment.  Like every
 * operator's, the result depends on the inputs alone (no atomics, a fixed order
 * of every sum), matrix by matrix: the others of a call do not change it.
 *
 * Conventions are those of ckpt_ops.h.
 */
#ifndef CKPT_MUON_H
#define CKPT_MUON_H

#include "ckpt_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The orthogonalisation of a matrix U [rows, cols]:
 *   X = U / (|U| + eps), |U| the 2-norm of its elements; its transpose where rows > cols
 *   `steps` times:  A = X X^T,  X = (a I + b A + c A A) X
 * which takes every singular value through the polynomial a x + b x^3 + c x^5
 * `steps` times and leaves the singular vectors as they are.  A matrix of
 * zeros stays zero; one with a NaN or an infinity becomes NaN altogether.
 * Operands of the products are held in 22 bits (two planes of fp16), sums in
 * fp32, the norm in fp64: X is as exact as with products in fp32 (1e-6 to
 * 5e-6), of any type, and in a step as well.  No value is held to less than
 * 2^-37, though: where eps is far above |U|, so that X begins small, it is off
 * by up to 2^-37 sqrt(rows cols) eps / |U| of itself (777 x 1003 with 1e4 |U|
 * for eps: 4e-5).  With a side of up to 16 all is held in fp64, and rounded
 * once (unless the most that a step multiplies a value by, to the power of
 * 2 (steps - 1), exceeds 1e7).
 */
typedef struct {
    uint32_t steps;       /* 1 to 64 */
    uint32_t reserved;    /* 0 */
    double a, b, c;       /* the polynomial, and all its iterates, stay within [-2, 2] on [0, 1] */
    double eps;           /* > 0 */
    uint64_t piece_bytes; /* bound on the workspace: matrices are taken in groups that fit (at least one);
                             0 = 4 GiB */
} ckpt_newton_schulz;

typedef struct {
    const void* in; /* [rows, cols], rows in_stride elements apart */
    uint64_t in_stride;
    void* out; /* may be `in` itself (with its stride) */
    uint64_t out_stride;
    uint64_t rows, cols; /* up to 2^22 each; 0 is allowed */
} ckpt_matrix;

/* Orthogonalises n matrices of one type (CKPT_TYPE_*).  `workspace`: 256-byte
 * aligned device memory of at least the bytes that _workspace says, the call's
 * own until its work on `stream` has run (NULL where that is 0).
 * Results lie in no element of each other or of other matrices (whose rows may
 * lie between theirs).  Errors: EINVAL (sizes, numbers, pointers, overlaps), EHIP. */
ckpt_status ckpt_orthogonalize_workspace(const ckpt_matrix* m, uint32_t n, const ckpt_newton_schulz* ns,
                                         uint64_t* bytes);
ckpt_status ckpt_orthogonalize(const ckpt_matrix* m, uint32_t n, uint32_t dtype, const ckpt_newton_schulz* ns,
                               int32_t device, void* workspace, uint64_t workspace_bytes, void* stream);

/* One matrix's fragments and its gradient, rows * cols elements each,
 * contiguous, of any alignment that is a whole number of elements. */
typedef struct {
    void* param; /* param_dtype: receives the rounded master copy */
    float* master;
    float* momentum;
    const void* grad; /* grad_dtype */
    uint64_t rows, cols;
    double scale; /* multiplies lr */
} ckpt_muon_matrix;

typedef struct {
    uint32_t param_dtype, grad_dtype; /* CKPT_TYPE_* */
    uint32_t nesterov, reserved;      /* 0 or 1; 0 */
    double lr, momentum, weight_decay; /* momentum in [0, 1) */
    const float* grad_scale;           /* device scalar or NULL (1) */
    ckpt_newton_schulz ns;
} ckpt_muon_args;

/* The step, in place, for n matrices: with g = *grad_scale * grad (1 if NULL),
 *   m = momentum m + (1 - momentum) g
 *   U = nesterov ? momentum m + (1 - momentum) g : m
 *   master = master (1 - lr weight_decay) - lr scale X,  X the orthogonalised U
 *   param = master rounded to nearest even.
 * Call it behind ckpt_wait(CKPT_WAIT_CAPTURED) on the same stream where a
 * snapshot of these fragments may be in flight.
 * Errors: EINVAL (also fragments that overlap, or have grad_scale in them), EHIP. */
ckpt_status ckpt_muon_workspace(const ckpt_muon_matrix* m, uint32_t n, const ckpt_muon_args* args, uint64_t* bytes);
ckpt_status ckpt_muon(const ckpt_muon_matrix* m, uint32_t n, const ckpt_muon_args* args, int32_t device,
                      void* workspace, uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CKPT_MUON_H */
