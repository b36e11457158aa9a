/*
 * libpnn, operators for sequence models: token embedding, gated linear recurrence, linear attention with
 * a decay for each head, norms around a block, and the losses that train towards a teacher's top logits
 * or by the model's own answers.
 *
 * A sequence model takes token ids through pnn_embed_fwd, runs pnn_scan_fwd or, in blocks between
 * pnn_norm_fwd, pnn_linattn_fwd along the sequence and is trained by pnn_distill_fwd_bwd or
 * pnn_policy_fwd_bwd; the _bwd entry points take the gradient back.  They need no
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
 *     batch, 2^20 heads and 2^30 steps of heads in a batch of linear attention and, where heads share
 *     keys, 2^32 pieces of four elements of their gradients, 2^30 heads of a norm's rows, 2^60
 *     elements from a tensor's first to its last).
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

/* ---- linear attention with a decay for each head ---------------------------------------------- */

/* strides of a [batch][length][heads][width] tensor, in elements */
typedef struct {
  int64_t batch; /* from sequence to sequence */
  int64_t step;  /* from step to step */
  int64_t head;  /* from head to head */
} pnn_head_stride;

typedef struct {
  int dtype;               /* pnn_dtype of q, k, v, o and their gradients */
  int64_t batch, length;
  int64_t heads;           /* of q and o */
  int64_t kv_heads;        /* of k and v: divides heads, head h takes k and v of h / (heads / kv_heads) */
  int64_t key_width;       /* elements of a head of q and k, 1 .. PNN_LINATTN_MAX_WIDTH */
  int64_t value_width;     /* elements of a head of v and o, likewise */
  pnn_head_stride q, k, v, o;           /* forward */
  pnn_head_stride dout, dq, dk, dv;     /* backward (not looked at by the forward) */
  float scale;
} pnn_linattn_desc;

#define PNN_LINATTN_MAX_WIDTH 256

/* Bytes of workspace of either direction (0: none, the pointer may be NULL). */
pnn_status pnn_linattn_sizes(const pnn_linattn_desc* d, size_t* forward, size_t* backward);

/* Per sequence and head, with lambda = exp(log_decay[head]):
 *     S_t = lambda S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t,   S_{-1} = s0 (zero when s0 is NULL)
 * log_decay: float[heads], each at most 0 (0: nothing is forgotten; -inf: all but the step's own term); one that is
 * positive or NaN makes its head's outputs NaN.  lengths as in pnn_scan_fwd: steps behind a sequence's end are not
 * looked at, their o is zero and they leave the state as it is.  s0, sT (nullable): float
 * [batch][heads][key_width][value_width], sT the state after the last step; may be s0 itself.  One step at a time
 * (length 1, sT = s0) is the form for answering.  o may not be q, k or v.  A q, k or v that is not finite makes
 * outputs of its own step and, for k and v, of later ones not finite (infinite or NaN), none of earlier steps.
 * bf16: products that a step's output is a sum of take the weighted q k and the state rounded to bf16, which makes
 * outputs about 2.4e-3 off where their own rounding is 1.7e-3; the state itself is a float sum, of terms kept to 24 bits
 * where sT (in the backward ds0) is wanted and to 16 where it only forms outputs. */
pnn_status pnn_linattn_fwd(const pnn_linattn_desc* d, const void* q, const void* k, const void* v,
                           const float* log_decay, const int32_t* lengths, const float* s0, void* o, float* sT,
                           void* workspace, void* stream);

/* The gradients, from dout and (nullable) dsT = dL/dsT, with Z_t = scale q_t dout_t^T + lambda Z_{t+1} and dsT (not
 * decayed) added at the last step:
 *     dq_t = scale S_t dout_t,   dk_t = Z_t v_t,   dv_t = Z_t^T k_t,   ds0 = lambda Z_0
 * dk and dv are summed over the heads that share them, in the heads' order.  log_decay has no gradient.  q, k, v, lengths
 * and s0 as in the forward; the states in between are formed again.  Steps behind a sequence's end get zero gradients.
 * ds0 (nullable) may be neither dsT nor s0.  dq, dk and dv may not be q, k, v, dout or one another. */
pnn_status pnn_linattn_bwd(const pnn_linattn_desc* d, const void* q, const void* k, const void* v,
                           const float* log_decay, const int32_t* lengths, const float* s0, const void* dout,
                           const float* dsT, void* dq, void* dk, void* dv, float* ds0, void* workspace, void* stream);

/* ---- norms before and after a block, with its gate and the residual sum ------------------------ */

/* strides of a [rows][heads][width] tensor, in elements */
typedef struct {
  int64_t row;  /* from row to row */
  int64_t head; /* from head to head */
} pnn_row_stride;

typedef struct {
  int dtype;               /* pnn_dtype of x, gate, res, h, y and their gradients; weights and their gradients are float */
  int64_t rows, heads;     /* a norm is over the width of one head of one row; 1 head: over the row */
  int64_t width;           /* 1 .. PNN_NORM_MAX_WIDTH */
  int post;                /* != 0: norm of the block's output x */
  int pre;                 /* != 0: norm of the sum h, the next block's input */
  pnn_row_stride x, gate, res, h, y;          /* forward (backward: x, gate and res or h) */
  pnn_row_stride dy, dh, dx, dgate, dres;     /* backward */
  float eps;               /* > 0 */
  float alpha;             /* scale of the block's output in the sum */
  int stored;              /* backward with pre: != 0: res is h as the forward stored it, 0: the residual */
} pnn_norm_desc;

#define PNN_NORM_MAX_WIDTH 16384

/* With norm(u) = u / sqrt(mean(u^2) + eps) over the width:
 *     a = post ? w_post norm(x) : x,   h = res + alpha a silu(gate),   y = w_pre norm(h)   (pre != 0)
 * w_post, w_pre: float[width], the same for every head (NULL: ones).  gate, res (NULL: without), h (NULL: not wanted,
 * with pre; may be res itself, with the same strides: the backward then takes it with `stored`), y (needed if pre != 0, not looked at otherwise).  y is formed from the sum
 * before it is rounded to h.  silu(-inf) is 0.  A row whose squares pass the float range is normed to zeros,
 * with no gradient through that norm. */
pnn_status pnn_norm_fwd(const pnn_norm_desc* d, const void* x, const float* w_post, const void* gate, const void* res,
                        const float* w_pre, void* h, void* y, void* stream);

/* Bytes of workspace for pnn_norm_bwd (needed if dw_post or dw_pre is wanted). */
pnn_status pnn_norm_workspace_size(const pnn_norm_desc* d, size_t* bytes);

/* The gradients, from dy (pre != 0) and (nullable) dh, the gradient that reaches h otherwise.  x, gate, w_post, w_pre as
 * in the forward.  res (looked at with pre only): the residual as in the forward (NULL: without), from which h is formed
 * again without its rounding, or, with `stored`, h as the forward stored it (h's strides; after a forward in place there
 * is nothing else): the gradients then are those at the stored h, whose rounding to bf16 is about 2e-3 of the weights'
 * gradients.  x is not looked at without post and gate where h is stored or pre is 0.  dres = dL/dres (nullable; may be
 * dh itself, with the same strides), dx, dgate (nullable).  dw_post, dw_pre (float[width], nullable): overwritten, or
 * added to with accumulate != 0; each sum has one order.  Without dres, dx, dgate and both weights' gradients nothing is
 * done. */
pnn_status pnn_norm_bwd(const pnn_norm_desc* d, const void* x, const float* w_post, const void* gate, const void* res,
                        const float* w_pre, const void* dy, const void* dh, void* dx, void* dgate, void* dres,
                        float* dw_post, float* dw_pre, int accumulate, void* workspace, void* stream);

/* ---- clipped policy loss with a KL term -------------------------------------------------------- */

typedef struct {
  int dtype;            /* pnn_dtype of logits and dlogits */
  int64_t rows, classes;
  int64_t logit_stride; /* elements from row to row of logits */
  int64_t grad_stride;  /* ... of dlogits */
  float temperature;    /* tau > 0 */
  float clip_low, clip_high; /* the ratio is held within 1 - clip_low .. 1 + clip_high; >= 0 */
  float kl;             /* weight of the KL term (0: ref is not looked at) */
  float scale;          /* factor of every gradient (1 / rows for a mean) */
} pnn_policy_desc;

/* For every row with a token a = tokens[row] >= 0, with p = softmax(logits / tau):
 *     l = log p_a,  r = exp(l - old),  x = ref - l
 *     loss = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl (exp(x) - 1 - x),   A = advantage
 *     dlogits_v = scale weight c / tau ([v = a] - p_v),   c = -[r A <= clip(r) A] r A - kl (exp(x) - 1)
 * logp (nullable): float[rows], l.  old (NULL: r = 1, with the gradient of r at 1), ref, weight (NULL: ones): float[rows].
 * The weight is a factor of the row's gradient, not of its loss.  r is infinite past the float range; with an advantage of
 * 0 there is no policy term all the same.  A row with a token below 0 (a prompt's, padding)
 * has loss, l and gradient 0 whatever the rest of it holds; a token not below `classes` makes them NaN.
 * loss: float[rows].  dlogits (nullable: loss and logp only) may be logits itself (with the same stride).
 * PNN_ERR_VALUE: tau not above zero, a clip bound below zero, or tau, log2(e) / tau, a bound, kl, scale or scale / tau
 * not finite. */
pnn_status pnn_policy_fwd_bwd(const pnn_policy_desc* d, const void* logits, const int32_t* tokens,
                              const float* advantage, const float* old, const float* ref, const float* weight,
                              float* loss, float* logp, void* dlogits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PNN_SEQ_H */
