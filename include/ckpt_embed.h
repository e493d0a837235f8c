/*
 * ckpt_embed.h -- C ABI of the vocabulary table's lookup and of its gradient:
 * the other end of a model whose head's losses are in ckpt_ops.h, with which
 * it may share the table.
 *
 * Every result depends on the inputs alone: a row's tokens are summed in their
 * order, in runs whose length the call's sizes decide (the number of tokens,
 * the rows' width and type, for few tokens also the number of words): columns
 * of a table by themselves need not have the bits of the whole table's.
 * Conventions are those of ckpt_ops.h.
 */
#ifndef CKPT_EMBED_H
#define CKPT_EMBED_H

#include "ckpt_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* tokens below 2^31 (0 is allowed), dim and vocab 1 to 2^22 */
typedef struct {
    uint32_t dtype;       /* CKPT_TYPE_* of the rows: out, and d_out */
    uint32_t table_dtype; /* of the table's: the lookup wants the rows' type */
    uint64_t tokens, dim, vocab;
    const int64_t* ids; /* [tokens] */
    int64_t ignore_index;
    double scale; /* a finite fp32 number once rounded */
    void* rows;   /* [tokens, dim], rows_stride elements apart: the lookup writes them, the gradient reads them */
    uint64_t rows_stride;
    void* table; /* [vocab, dim]: the lookup reads it; the gradient writes it, or adds to it */
    uint64_t table_stride;
                  /* rows and table: not in one another, from the first to the last element of each */
    uint32_t add; /* the gradient: 0 = every row is written, 1 = added to what is there */
    uint32_t reserved; /* 0 */
} ckpt_embed_args;

/* rows[t] = scale * table[ids[t]], rounded once.  A token whose id is
 * ignore_index has a row of zeros; one with another id outside [0, vocab) a
 * row of NaN.  Errors: EINVAL (sizes, strides below a row, null or foreign
 * pointers), EHIP. */
ckpt_status ckpt_embedding(const ckpt_embed_args* a, int32_t device, void* stream);

/* table[v] = (add ? table[v] : 0) + scale * sum of rows[t] over the tokens with
 * ids[t] == v, summed in fp32 and rounded once.  Tokens with ignore_index or an
 * id outside [0, vocab) give nothing and are not read.  With `add` rows that no
 * token has are left as they are.  `workspace`: 256-byte aligned device
 * memory of at least the bytes that _workspace says, the call's own until its
 * work on `stream` has run (NULL where that is 0).  Errors as above. */
ckpt_status ckpt_embedding_grad_workspace(const ckpt_embed_args* a, uint64_t* bytes);
ckpt_status ckpt_embedding_grad(const ckpt_embed_args* a, int32_t device, void* workspace, uint64_t workspace_bytes,
                                void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CKPT_EMBED_H */
