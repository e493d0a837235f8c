/*
 * ckpt_ops.h -- C ABI of the training-step operators of libckpt: the losses
 * of the vocabulary head with their gradients, and the clipped optimizer step
 * over the state's fragments.
 *
 * They are the two ends of the step that the snapshots of ckpt.h protect
 * (paper Sec. VI-A: the wait before the optimizer step): the loss makes the
 * gradient without holding the logits of all tokens in HBM, which the
 * snapshot's device image has a use for, and the optimizer step is what the
 * gate keeps off fragments that are not captured yet.  Every result depends
 * on the inputs alone (no atomics, a fixed order of every sum), so a run
 * restored from a snapshot repeats the lost steps bit for bit.
 *
 * Conventions are those of ckpt.h: status codes, streams as void*, nothing
 * thrown, and ckpt_last_error(NULL) for the text of this thread's last
 * failure.  A call enqueues its work on `stream` and returns without waiting;
 * it allocates nothing, keeps nothing between calls, and records no memset or
 * copy node (it may be captured into a HIP graph).  What its pointers name has
 * to stay until that work has run.  Device pointers are checked on the host
 * against their allocations; what device memory holds (targets, indices) is
 * not.
 */
#ifndef CKPT_OPS_H
#define CKPT_OPS_H

#include "ckpt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types (the tags a fragment table may carry) */
#define CKPT_TYPE_BF16 1
#define CKPT_TYPE_F32 2

#define CKPT_LOSS_MEAN 0 /* the weighted mean over the tokens that count */
#define CKPT_LOSS_SUM 1

/* ---- Losses of the vocabulary head ----
 *
 * The logits l = hidden weight^T are never held for more than one piece of the
 * tokens; the cross entropy without gradients holds none.  With w the token weight, lse = log sum_v exp l_v and y the target:
 *   ce_n   = lse_n - l_n,y
 * and, with topk > 0 and alpha > 0, from a teacher's logits t_k at the words i_k:
 *   q      = softmax of t / T over the row's entries
 *   kd_n   = T^2 sum_k q_k (log q_k - l_n,i_k / T + lse^T_n),  lse^T = log sum_v exp(l_v / T)
 *   loss_n = alpha kd_n + (1 - alpha) ce_n
 * (loss_n = ce_n with topk == 0 or alpha == 0: the teacher's entries are then
 * not read).  The loss is sum_n w_n loss_n, divided by
 * the sum of w_n over the rows that count for CKPT_LOSS_MEAN (0 where none
 * does).  The gradients are those of grad_scale * loss.
 *
 * Which rows count: one whose target is not ignore_index (where the cross
 * entropy has a share: topk == 0 or alpha < 1), or that has a teacher entry
 * (where the teacher has one: topk > 0 and alpha > 0); never one of weight 0.  Rows that do not count are not read: whatever
 * `hidden` holds there, NaN included, their loss, log-sum-exp and gradient
 * are 0.  A target outside [0, vocab) other than ignore_index, or a teacher
 * index >= vocab, makes the row's loss and gradient NaN.  A teacher index below 0 marks an
 * entry that is absent, and so does a logit of -inf; a row without entries
 * has no kd.  The same word may be given twice.
 */
typedef struct {
    uint32_t dtype;     /* CKPT_TYPE_*: hidden, weight and their gradients */
    uint32_t reduction; /* CKPT_LOSS_* */
    uint64_t tokens, dim, vocab; /* tokens below 2^31 (0 is allowed), the others 1 to 2^22 */
    const void* hidden; /* [tokens, dim], rows hidden_stride elements apart */
    uint64_t hidden_stride;
    const void* weight; /* [vocab, dim] */
    uint64_t weight_stride;
    const int64_t* target; /* [tokens]; NULL where the cross entropy has no share */
    int64_t ignore_index;
    const float* token_weight; /* [tokens] or NULL (1 for each) */
    uint32_t topk;             /* teacher entries a token, at most 1024; 0 = cross entropy alone */
    uint32_t teacher_dtype;    /* CKPT_TYPE_* of teacher_logits */
    const int64_t* teacher_index; /* [tokens, topk] */
    uint64_t teacher_index_stride;
    const void* teacher_logits; /* [tokens, topk] */
    uint64_t teacher_logits_stride;
    float temperature, alpha; /* T > 0, 1/T and T^2 within fp32; alpha in [0, 1] */
    const float* grad_scale;  /* device scalar or NULL (1) */
    uint64_t piece_bytes;     /* bound on what is held for the tokens at a time: their logits and the logits'
                                 gradient, their copy and statistics, the sums of d_hidden where it is cut; at least
                                 what 256 tokens take without the last; 0 = 2 GiB.  Not in it: 4 bytes a token, copies
                                 of weight, the running d_weight of several pieces */
    /* outputs */
    float* loss;       /* scalar */
    float* token_loss; /* [tokens] loss_n, before the weight */
    float* lse;        /* [tokens] lse (topk > 0 and alpha > 0: lse^T) */
    void* d_hidden;    /* [tokens, dim]; both gradients or neither (NULL) */
    uint64_t d_hidden_stride;
    void* d_weight; /* [vocab, dim] */
    uint64_t d_weight_stride;
} ckpt_linear_loss_args;

/* Device memory the call works in, for these sizes, strides and pointers (an
 * operand's alignment decides whether it is copied).  Errors: EINVAL (sizes,
 * numbers, strides whose rows lie beyond 64 bits of bytes). */
ckpt_status ckpt_linear_loss_workspace(const ckpt_linear_loss_args* a, uint64_t* bytes);

/* The loss and, where d_hidden and d_weight are given, its gradients.
 * `workspace`: 256-byte aligned device memory of at least the bytes above,
 * the call's own until its work on `stream` has run.
 * Errors: EINVAL (sizes, strides below a row, a null or foreign pointer, a
 * misaligned one, outputs that are NULL one by one), EHIP (a launch). */
ckpt_status ckpt_linear_loss(const ckpt_linear_loss_args* a, int32_t device, void* workspace,
                             uint64_t workspace_bytes, void* stream);

/* ---- The optimizer step ----
 *
 * ckpt_grad_norm: out[0] = the 2-norm of all elements of the fragments,
 * out[1] = min(1, max_norm / (out[0] + 1e-6)), 1 where max_norm <= 0.
 * grads[k].nbytes is a whole number of elements of `dtype`; no alignment but
 * the element's is needed.  `scratch`: CKPT_GRAD_NORM_SCRATCH bytes, 8-byte
 * aligned.  Errors: EINVAL, EHIP. */
#define CKPT_GRAD_NORM_SCRATCH 16384
ckpt_status ckpt_grad_norm(const ckpt_tensor* grads, uint32_t n, uint32_t dtype, float max_norm, float* out,
                           void* scratch, int32_t device, void* stream);

/* One parameter's four fragments and its gradient, numel elements each; any
 * alignment that is a whole number of elements. */
typedef struct {
    void* param;       /* param_dtype: receives the rounded master copy */
    float* master;
    float* exp_avg;
    float* exp_avg_sq;
    const void* grad;  /* grad_dtype */
    uint64_t numel;    /* 0 is allowed */
} ckpt_adamw_fragment;

/* AdamW, in place, for n parameters: with g = *grad_scale * grad (1 if NULL),
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   master = master (1 - lr weight_decay)
 *            - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps),
 *   param = master rounded to nearest even.
 * step >= 1.  Call it behind ckpt_wait(CKPT_WAIT_CAPTURED) on the same stream
 * where a snapshot of these fragments may be in flight.
 * Errors: EINVAL, EHIP. */
ckpt_status ckpt_adamw(const ckpt_adamw_fragment* f, uint32_t n, uint32_t param_dtype, uint32_t grad_dtype,
                       uint64_t step, double lr, double beta1, double beta2, double eps, double weight_decay,
                       const float* grad_scale, int32_t device, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CKPT_OPS_H */
