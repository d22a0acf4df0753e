/*
 * symb_loss.h -- where a fine-tuning client's backward pass starts: its loss through the frozen vocabulary matrix that all clients share, and the gradient of the rows that
 * went in, for the whole flattened batch.  The logits are never in memory: the largest thing that a call holds is the weights of a few thousand rows (symb_loss_workspace_bytes).
 *
 * Types, ownership, ordering and errors are symb.h's: bf16 activations and weights, DEVICE tensors owned by the caller, 16-byte aligned unless said otherwise, HOST descriptors copied during the
 * call, everything enqueued on `stream`, all checks before the first launch.  A batch without rows is legal; its losses are zeros.  A call's descriptors (12 bytes a segment) fill one slot of 2 MiB.
 *
 * For a row x of segment i and a vocabulary of V tokens
 *     s_v = x . W_v,   z_v = s_v  (cap > 0: cap tanh(s_v / cap))
 *   symb_cross_entropy    L = log sum_v exp(z_v) - z_label
 *   symb_distillation     q = softmax over the row's entries j of (logit_j / T_i),  p = softmax over all v of (z_v / T_i),
 *                         L = T_i^2 sum_j q_j (log q_j - log p[id_j]),   terms with q_j = 0 left out
 * A row with a negative label, or without any entry of an id >= 0, takes no part: its loss and its gradient are zeros, and what its x holds is not looked at.  (An entry with a negative id is absent.)
 *   loss_i   mean (SYMB_LOSS_SUM: sum) of L over the segment's rows that take part; 0 if none does
 *   dX       scale_i d loss_i / dx
 * A label or id of V or more is never followed: the row's loss and gradient are NaN, and so are those of a row with a score of NaN or +infinity, or of -infinity at its label or its teacher's best entry,
 * or with a logit of NaN or +infinity (-infinity beside others: a share of zero); no other row's.  A token that a row names twice counts with the sum of its shares.
 * What is rounded: the weights p_v - q_v enter the gradient's product as bf16, off by 2^-8 of each at most (in batches of up to 64 rows as two bf16 terms, 2^-16); dX is rounded once.  Scores, sums and
 * losses are fp32, a label's own score is formed in 64 bits: a sure row's loss (p_label near one) keeps its relative precision.  Capping is good to 2^-21 of a score.
 * Deterministic: the same arguments give the same bits.  What else is in the batch can change a row's loss and gradient in the last rounding.
 */
#ifndef SYMB_LOSS_H
#define SYMB_LOSS_H

#include "symb.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SYMB_LOSS_MEAN = 0, SYMB_LOSS_SUM = 1 } symb_loss_reduction;

typedef struct {
    float scale;                   /* of the gradient: what d (what the client minimises) / d loss_i is.  Finite */
    float temperature;             /* T_i of symb_distillation: positive, finite (2^-20 to 2^20; others: SYMB_ERR_UNSUPPORTED); not looked at by symb_cross_entropy */
} symb_loss;

typedef struct {
    int32_t width;                 /* d: a multiple of 8, at most SYMB_LOSS_MAX_WIDTH */
    int32_t vocab;                 /* V: any number from 1 to SYMB_LOSS_MAX_VOCAB */
    int32_t num_segments;
    const int32_t* seg_offsets;    /* HOST, as in symb_batch.  T rows: at most SYMB_LOSS_MAX_ROWS, and T times width below 2^31 (SYMB_ERR_UNSUPPORTED otherwise: give more in several calls) */
    const symb_loss* losses;       /* HOST, num_segments entries */
    int32_t reduction;             /* symb_loss_reduction */
    float cap;                     /* >= 0, finite; 0: scores as they are */
} symb_loss_batch;

enum { SYMB_LOSS_MAX_WIDTH = 32768, SYMB_LOSS_MAX_VOCAB = 1 << 22, SYMB_LOSS_MAX_ENTRIES = 1024, SYMB_LOSS_MAX_ROWS = 1 << 22 };

/* Bytes of workspace for a call on this batch: entries 0 for symb_cross_entropy, else the entries of symb_distillation; gradient 0 for losses alone (dX NULL).  Host-only. */
symb_status symb_loss_workspace_bytes(const symb_loss_batch* b, int32_t entries, int32_t gradient, size_t* out);

/* X [T][width] bf16, W [vocab][width] bf16, dense rows; labels [T] int32 (4-byte aligned).
 * loss [num_segments] fp32 or NULL, row_loss [T] fp32 or NULL (both 4-byte aligned), dX [T][width] bf16 or NULL (losses alone); dX may be X. */
symb_status symb_cross_entropy(symb_handle h, const symb_loss_batch* b, const void* X, const void* W, const int32_t* labels, float* loss, float* row_loss, void* dX,
                               void* ws, size_t ws_bytes, void* stream);

/* ids [T][entries] int32, logits [T][entries] fp32 (both 4-byte aligned): the teacher's entries of every row, in any order; 1 <= entries <= SYMB_LOSS_MAX_ENTRIES.  The rest as above. */
symb_status symb_distillation(symb_handle h, const symb_loss_batch* b, const void* X, const void* W, const int32_t* ids, const float* logits, int32_t entries, float* loss,
                              float* row_loss, void* dX, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SYMB_LOSS_H */
