/*
 * libpnn, operators for sequence models: token embedding, gated linear recurrence, and the loss that
 * trains towards a teacher's top logits.
 *
 * A sequence model takes token ids through pnn_embed_fwd, runs pnn_scan_fwd along the sequence and is
 * trained by pnn_distill_fwd_bwd; pnn_scan_bwd and pnn_embed_bwd take the gradient back.  They need no
 * plan: each call takes a description of its tensors (filled once, reusable) and device pointers.
 *
 * Conventions for every entry point (as in pnn.h, except for alignment)
 *   - Every tensor pointer is a DEVICE pointer owned by the caller.  Entry points never allocate
 *     memory, free or synchronise; all work is ordered on the given stream and can be captured into
 *     a HIP graph.  Nothing is kept between calls: a workspace holds nothing a later call needs, and
 *     needs no initialisation.  Calls that share a workspace must not overlap in time.
 *   - Element types are pnn_dtype (float or bfloat16 bit patterns); arithmetic, sums and recurrent
 *     states are fp32, results are rounded to nearest even once, where they are stored.
 *   - The elements of a row (a token's width, a step's channels, a sample's classes) are contiguous;
 *     everything above that has a stride in elements.  Strides may not be negative; those of an
 *     output must keep its rows apart (PNN_ERR_SHAPE).
 *   - Alignment: tensors to their element, workspaces to 256 bytes (PNN_ERR_ALIGN).  Rows that start
 *     on 16-byte boundaries (pointer and strides) are moved in 16-byte pieces and run fastest.
 *   - An index (token, class) below zero means "none"; one past the end is the caller's mistake and
 *     turns the row it belongs to into NaN.
 *   - An output shares no element with an input, a workspace or another output, unless its entry point
 *     says that it may stand in an input's place.  Equal pointers are refused (PNN_ERR_SHAPE); whether
 *     tensors overlap otherwise is not looked at.
 *   - Empty problems are valid (pointers of tensors without elements may be NULL).
 *   - Results do not depend on timing: no sum is formed in an order that varies from run to run.
 *   - Return value: PNN_OK or a negative pnn_status; on error nothing has been enqueued, except for
 *     PNN_ERR_HIP.  PNN_ERR_TOO_LARGE: sizes or offsets beyond what the kernels index (2^28 samples,
 *     2^22 pieces of 32 tokens x 64 elements, 32 table rows or 16384 elements
 *     of the table, 2^31 - 1 classes, 2^30 steps, 2^21 times 64 channels in a
 *     batch, 2^60 elements from a tensor's first to its last).
 */
#ifndef PNN_SEQ_H
#define PNN_SEQ_H

#include "pnn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- token embedding ------------------------------------------------------------------------ */

typedef struct {
  int dtype;            /* pnn_dtype of the rows (out, dout) */
  int table_dtype;      /* pnn_dtype of the table; its gradient is float whatever this is */
  int token_bytes;      /* 4: int32 tokens, 8: int64 tokens (contiguous) */
  int64_t n;            /* tokens */
  int64_t vocab;        /* rows of the table */
  int64_t width;        /* elements of a row */
  int64_t table_stride; /* elements from row to row of the table and of its gradient */
  int64_t row_stride;   /* elements from row to row of out / dout */
  float scale;
} pnn_embed_desc;

/* out[i] = scale * table[tokens[i]]; zeros for a token below 0, NaN for one not below vocab.
 * PNN_ERR_VALUE (also below): scale not finite. */
pnn_status pnn_embed_fwd(const pnn_embed_desc* d, const void* table, const void* tokens, void* out,
                         void* stream);

/* Bytes of workspace for pnn_embed_bwd. */
pnn_status pnn_embed_workspace_size(const pnn_embed_desc* d, size_t* bytes);

/* dtable[v] = scale * sum over the tokens i with tokens[i] = v of dout[i], for every row v (rows
 * without tokens become zero); with accumulate != 0 the sum is added to dtable[v] and rows without
 * tokens are left as they are.  Tokens outside the table have no gradient.  The tokens are sorted
 * (stably, on the device) and a row's sum has one order whatever the run: in token order within tiles of
 * sorted tokens, the tiles' sums in a fixed order after that. */
pnn_status pnn_embed_bwd(const pnn_embed_desc* d, const void* dout, const void* tokens, float* dtable,
                         int accumulate, void* workspace, void* stream);

/* ---- gated linear recurrence ----------------------------------------------------------------- */

/* strides of a [batch][length][channels] tensor, in elements */
typedef struct {
  int64_t batch; /* from sequence to sequence */
  int64_t step;  /* from step to step */
} pnn_seq_stride;

typedef struct {
  int dtype;                 /* pnn_dtype of x, gate, h and their gradients */
  int64_t batch, length, channels;
  pnn_seq_stride x, gate, h; /* forward */
  pnn_seq_stride dh, dx, dgate; /* backward (not looked at by the forward) */
} pnn_scan_desc;

/* Bytes of `states` (what the forward keeps for the backward) and of the workspace either direction
 * needs (0: none, the pointer may be NULL). */
pnn_status pnn_scan_sizes(const pnn_scan_desc* d, size_t* states, size_t* workspace);

/* Per sequence and channel, with f_t = sigmoid(gate_t):
 *     h_t = f_t h_{t-1} + (1 - f_t) x_t,   h_{-1} = h0 (zero when h0 is NULL)
 * lengths (int32[batch], nullable): steps t >= lengths[b] are not part of sequence b: their x and gate
 * are ignored, their h is zero and they leave the state as it is (values outside 0 .. length count as
 * the nearer end).  hT (nullable, float [batch][channels]): the state after the last step; may be h0
 * itself.  states (nullable): kept for pnn_scan_bwd.  h0: float [batch][channels].
 * One step at a time (length 1, hT = h0) is the form for answering: the state stays in place.
 * h may not be x or gate.  f_t or 1 - f_t is 0 where it is below about 1.6e-38.  A state that is not
 * finite makes what follows it in its sequence and channel not finite (infinite or NaN). */
pnn_status pnn_scan_fwd(const pnn_scan_desc* d, const void* x, const void* gate, const int32_t* lengths,
                        const float* h0, void* h, float* hT, float* states, void* workspace, void* stream);

/* The gradients, from dh and (nullable) dhT = dL/dhT, with G_t = dh_t + f_{t+1} G_{t+1} and dhT beyond
 * the last step:
 *     dx_t = (1 - f_t) G_t,   dgate_t = G_t (h_{t-1} - x_t) f_t (1 - f_t),   dh0 = f_0 G_0
 * x, gate, lengths as in the forward that filled `states` (h itself is not needed: the states in
 * between are formed again).  Steps beyond a sequence's length get zero gradients.  dh0 (nullable):
 * float [batch][channels]; may be dhT itself.  dx and dgate may not be x, gate, dh or one another. */
pnn_status pnn_scan_bwd(const pnn_scan_desc* d, const void* x, const void* gate, const int32_t* lengths,
                        const float* states, const void* dh, const float* dhT, void* dx, void* dgate,
                        float* dh0, void* workspace, void* stream);

/* ---- distillation from a teacher's top logits ------------------------------------------------- */

typedef struct {
  int dtype;            /* pnn_dtype of logits and dlogits */
  int teacher_dtype;    /* pnn_dtype of the teacher's logits */
  int64_t rows, classes;
  int64_t top;          /* teacher entries of a row, 0 .. PNN_DISTILL_MAX_TOP */
  int64_t logit_stride; /* elements from row to row of logits */
  int64_t grad_stride;  /* ... of dlogits */
  int64_t top_stride;   /* ... of the teacher's logits and of index */
  float temperature;    /* tau > 0 */
  float alpha;          /* weight of the teacher's term; 1 - alpha: weight of the labels' */
  float scale;          /* factor of every gradient (1 / rows for a mean) */
} pnn_distill_desc;

#define PNN_DISTILL_MAX_TOP 1024

/* For every row, with q = softmax(logits / tau), s = softmax(logits) and p = softmax(teacher / tau) over
 * the row's entries k with index[k] >= 0:
 *     loss = alpha tau^2 sum_k p_k (log p_k - log q_{index_k})  +  (1 - alpha) (-log s_label)
 *     dlogits_v = scale weight (alpha tau (q_v - sum_{k: index_k = v} p_k) + (1 - alpha) (s_v - [v = label]))
 * The first term is zero for a row without entries (all indices below 0, or all its logits -inf), the
 * second without labels (NULL) or for a label below 0; a term whose weight (alpha, 1 - alpha) is 0 is
 * left out, its indices or labels unread.  An entry whose p is 0 adds nothing.  A class
 * may stand in several entries.  An index or label not below `classes` makes the row's loss and
 * gradient NaN.  weight (float[rows], nullable): factor of the row's gradient, not of its loss.
 * loss: float[rows].  dlogits (nullable: loss only) may be logits itself (with the same stride).
 * PNN_ERR_VALUE: tau not above zero, or tau, log2(e) / tau, alpha tau^2 or scale not finite. */
pnn_status pnn_distill_fwd_bwd(const pnn_distill_desc* d, const void* logits, const int32_t* index,
                               const void* teacher, const int32_t* labels, const float* weight, float* loss,
                               void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PNN_SEQ_H */
