// Entry points of the sequence operators (pnn_seq.h): argument checks, then the launchers.
#include <math.h>

#include <initializer_list>

#include "pnn_seq.h"
#include "seq_internal.h"

using namespace pnn;

namespace {

constexpr int64_t MAX_COUNT = 0x7fffffff;
constexpr int64_t MAX_SPAN = int64_t(1) << 60;

bool type_ok(int t) { return t == PNN_F32 || t == PNN_BF16; }
int type_size(int t) { return t == PNN_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// whether an output starts where another one or an input does; NULL: a tensor that the call does not look at
bool meet(std::initializer_list<const void*> out, std::initializer_list<const void*> in) {
  for (auto o = out.begin(); o != out.end(); ++o) {
    if (*o == nullptr) continue;
    for (auto p = o + 1; p != out.end(); ++p)
      if (*p == *o) return true;
    for (const void* p : in)
      if (p == *o) return true;
  }
  return false;
}

// elements from the first to the last of `rows` rows of `width`, `stride` apart; < 0: too many
int64_t span(int64_t rows, int64_t stride, int64_t width) {
  const __int128 v = rows > 0 ? (__int128)(rows - 1) * stride + width : 0;
  return v > (__int128)MAX_SPAN ? -1 : (int64_t)v;
}

pnn_status rows_ok(int64_t rows, int64_t stride, int64_t width, bool out) {
  if (stride < 0 || (out && rows > 1 && stride < width)) return PNN_ERR_SHAPE;
  return span(rows, stride, width) < 0 ? PNN_ERR_TOO_LARGE : PNN_OK;
}

// a [batch][length][channels] tensor: strides, and of an output that no two rows share an element
// (sequences outside steps or steps outside sequences; interleaved rows are refused)
pnn_status seq_ok(const pnn_scan_desc* d, const pnn_seq_stride& s, bool out) {
  if (s.batch < 0 || s.step < 0) return PNN_ERR_SHAPE;
  const __int128 steps = (__int128)(d->length - 1) * s.step, seqs = (__int128)(d->batch - 1) * s.batch;
  if (steps + seqs + d->channels > (__int128)MAX_SPAN) return PNN_ERR_TOO_LARGE;
  if (out) {
    const bool step_ok = d->length <= 1 || s.step >= d->channels, batch_ok = d->batch <= 1 || s.batch >= d->channels;
    if (!step_ok || !batch_ok) return PNN_ERR_SHAPE;
    if (d->length > 1 && d->batch > 1 && s.batch < steps + d->channels && s.step < seqs + d->channels)
      return PNN_ERR_SHAPE;
  }
  return PNN_OK;
}

pnn_status embed_ok(const pnn_embed_desc* d) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype) || !type_ok(d->table_dtype) || (d->token_bytes != 4 && d->token_bytes != 8))
    return PNN_ERR_DTYPE;
  if (d->n < 0 || d->vocab < 0 || d->width < 0) return PNN_ERR_SHAPE;
  // grids: at most a workgroup for every 32 tokens x 64 elements, for every 32 rows and for every 16384 elements of the table
  if (d->n > (1 << 28) || d->vocab >= MAX_COUNT || d->width > (1 << 23)) return PNN_ERR_TOO_LARGE;
  if (cdiv64(d->n, 32) * cdiv64(d->width, 64) + cdiv64(d->vocab, 32) + cdiv64(d->vocab * d->width, 16384) > (1 << 22)) return PNN_ERR_TOO_LARGE;
  if (pnn_status e = rows_ok(d->vocab, d->table_stride, d->width, false)) return e;
  if (pnn_status e = rows_ok(d->n, d->row_stride, d->width, false)) return e;
  if (!isfinite(d->scale)) return PNN_ERR_VALUE;
  return PNN_OK;
}

pnn_status scan_ok(const pnn_scan_desc* d) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype)) return PNN_ERR_DTYPE;
  if (d->batch < 0 || d->length < 0 || d->channels < 0) return PNN_ERR_SHAPE;
  if (d->batch > MAX_COUNT || d->length > (1 << 30) || d->channels > MAX_COUNT) return PNN_ERR_TOO_LARGE;
  // a launch has up to 1024 threads for every 64 channels of a sequence, and the states are held densely
  if (cdiv64(d->channels, 64) * d->batch > (1 << 21) || (__int128)d->batch * d->channels * d->length > (__int128)MAX_SPAN)
    return PNN_ERR_TOO_LARGE;
  return PNN_OK;
}

// a [batch][length][heads][width] tensor, as seq_ok: of an output, each stride in ascending order holds all that is
// inside it
pnn_status heads_ok(const pnn_linattn_desc* d, const pnn_head_stride& s, int64_t heads, int64_t width, bool out) {
  if (s.batch < 0 || s.step < 0 || s.head < 0) return PNN_ERR_SHAPE;
  int64_t count[3] = {d->batch, d->length, heads}, stride[3] = {s.batch, s.step, s.head};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      if (stride[j] > stride[j + 1]) {
        const int64_t c = count[j], t = stride[j];
        count[j] = count[j + 1], stride[j] = stride[j + 1];
        count[j + 1] = c, stride[j + 1] = t;
      }
  __int128 inside = width;
  for (int i = 0; i < 3; ++i) {
    if (count[i] <= 1) continue;
    if (out && stride[i] < inside) return PNN_ERR_SHAPE;
    inside += (__int128)(count[i] - 1) * stride[i];
    if (inside > (__int128)MAX_SPAN) return PNN_ERR_TOO_LARGE;
  }
  return PNN_OK;
}

pnn_status linattn_ok(const pnn_linattn_desc* d) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype)) return PNN_ERR_DTYPE;
  if (d->batch < 0 || d->length < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0 ||
      d->key_width < 1 || d->value_width < 1)
    return PNN_ERR_SHAPE;
  if (d->key_width > LIN_MAX_WIDTH || d->value_width > LIN_MAX_WIDTH || d->length > (1 << 30) || d->heads > (1 << 20) ||
      d->batch > (1 << 20) || d->batch * d->heads > (1 << 20) ||
      (__int128)d->batch * d->heads * d->length > ((__int128)1 << 30))
    return PNN_ERR_TOO_LARGE;
  if (!isfinite(d->scale)) return PNN_ERR_VALUE;
  return PNN_OK;
}

pnn_status linattn_in_ok(const pnn_linattn_desc* d) {
  if (pnn_status e = heads_ok(d, d->q, d->heads, d->key_width, false)) return e;
  if (pnn_status e = heads_ok(d, d->k, d->kv_heads, d->key_width, false)) return e;
  return heads_ok(d, d->v, d->kv_heads, d->value_width, false);
}

// a [rows][heads][width] tensor; rows outside heads or heads outside rows
pnn_status norm_rows_ok(const pnn_norm_desc* d, const pnn_row_stride& s, bool out) {
  if (s.row < 0 || s.head < 0) return PNN_ERR_SHAPE;
  const __int128 rows = (__int128)(d->rows - 1) * s.row, heads = (__int128)(d->heads - 1) * s.head;
  if (rows + heads + d->width > (__int128)MAX_SPAN) return PNN_ERR_TOO_LARGE;
  if (out) {
    if ((d->rows > 1 && s.row < d->width) || (d->heads > 1 && s.head < d->width)) return PNN_ERR_SHAPE;
    if (d->rows > 1 && d->heads > 1 && s.row < heads + d->width && s.head < rows + d->width) return PNN_ERR_SHAPE;
  }
  return PNN_OK;
}

// whether two tensors that start in one place are the same elements
bool same(const pnn_row_stride& a, const pnn_row_stride& b, const pnn_norm_desc* d) {
  return (d->rows <= 1 || a.row == b.row) && (d->heads <= 1 || a.head == b.head);
}

pnn_status norm_ok(const pnn_norm_desc* d) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype)) return PNN_ERR_DTYPE;
  if (d->rows < 0 || d->heads < 1 || d->width < 1) return PNN_ERR_SHAPE;
  // rows are counted in 32 bits, with a step of all teams (up to 2048 x 16) beyond the last
  if (d->width > PNN_NORM_MAX_WIDTH || d->rows > (1 << 30) || d->heads > (1 << 30) || d->rows * d->heads > (1 << 30))
    return PNN_ERR_TOO_LARGE;
  if (!isfinite(d->eps) || !(d->eps >= 1e-37f) || !isfinite(d->alpha)) return PNN_ERR_VALUE;
  return PNN_OK;
}

}  // namespace

extern "C" {

pnn_status pnn_embed_fwd(const pnn_embed_desc* d, const void* table, const void* tokens, void* out, void* stream) {
  if (pnn_status e = embed_ok(d)) return e;
  if (pnn_status e = rows_ok(d->n, d->row_stride, d->width, true)) return e;
  if (d->n == 0 || d->width == 0) return PNN_OK;
  if ((table == nullptr && d->vocab > 0) || tokens == nullptr || out == nullptr) return PNN_ERR_NULL;
  if (!aligned(table, type_size(d->table_dtype)) || !aligned(tokens, d->token_bytes) ||
      !aligned(out, type_size(d->dtype)))
    return PNN_ERR_ALIGN;
  if (out == table) return PNN_ERR_SHAPE;
  return launch_embed_fwd(*d, table, tokens, out, (hipStream_t)stream) ? PNN_ERR_HIP : PNN_OK;
}

pnn_status pnn_embed_workspace_size(const pnn_embed_desc* d, size_t* bytes) {
  if (bytes == nullptr) return PNN_ERR_NULL;
  if (pnn_status e = embed_ok(d)) return e;
  *bytes = (size_t)embed_ws(*d).bytes;
  return PNN_OK;
}

pnn_status pnn_embed_bwd(const pnn_embed_desc* d, const void* dout, const void* tokens, float* dtable, int accumulate,
                         void* workspace, void* stream) {
  if (pnn_status e = embed_ok(d)) return e;
  if (pnn_status e = rows_ok(d->vocab, d->table_stride, d->width, true)) return e;
  if (d->vocab == 0 || d->width == 0) return PNN_OK;
  if (dtable == nullptr || (d->n > 0 && (dout == nullptr || tokens == nullptr || workspace == nullptr)))
    return PNN_ERR_NULL;
  if (!aligned(dtable, 4) || !aligned(dout, type_size(d->dtype)) || !aligned(tokens, d->token_bytes) ||
      !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  if ((const void*)dtable == dout) return PNN_ERR_SHAPE;
  return launch_embed_bwd(*d, dout, tokens, dtable, accumulate, workspace, (hipStream_t)stream) ? PNN_ERR_HIP : PNN_OK;
}

pnn_status pnn_scan_sizes(const pnn_scan_desc* d, size_t* states, size_t* workspace) {
  if (states == nullptr || workspace == nullptr) return PNN_ERR_NULL;
  if (pnn_status e = scan_ok(d)) return e;
  *states = (size_t)(d->batch * scan_chunks(*d) * d->channels * 4);
  *workspace = (size_t)scan_ws_bytes(*d);
  return PNN_OK;
}

pnn_status pnn_scan_fwd(const pnn_scan_desc* d, const void* x, const void* gate, const int32_t* lengths,
                        const float* h0, void* h, float* hT, float* states, void* workspace, void* stream) {
  if (pnn_status e = scan_ok(d)) return e;
  if (pnn_status e = seq_ok(d, d->x, false)) return e;
  if (pnn_status e = seq_ok(d, d->gate, false)) return e;
  if (pnn_status e = seq_ok(d, d->h, true)) return e;
  if (d->batch == 0 || d->channels == 0) return PNN_OK;
  if (d->length > 0 && (x == nullptr || gate == nullptr || h == nullptr)) return PNN_ERR_NULL;
  if (workspace == nullptr && scan_ws_bytes(*d) > 0) return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(x, es) || !aligned(gate, es) || !aligned(h, es) || !aligned(lengths, 4) || !aligned(h0, 4) ||
      !aligned(hT, 4) || !aligned(states, 4) || !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  if (d->length > 0 && (h == x || h == gate)) return PNN_ERR_SHAPE;
  ScanArgs a = {};
  a.x = x;
  a.gate = gate;
  a.lengths = lengths;
  a.h0 = h0;
  a.h = h;
  a.hT = hT;
  a.states = states;
  a.ws = workspace;
  return launch_scan_fwd(*d, a, (hipStream_t)stream) ? PNN_ERR_HIP : PNN_OK;
}

pnn_status pnn_scan_bwd(const pnn_scan_desc* d, const void* x, const void* gate, const int32_t* lengths,
                        const float* states, const void* dh, const float* dhT, void* dx, void* dgate, float* dh0,
                        void* workspace, void* stream) {
  if (pnn_status e = scan_ok(d)) return e;
  if (pnn_status e = seq_ok(d, d->x, false)) return e;
  if (pnn_status e = seq_ok(d, d->gate, false)) return e;
  if (pnn_status e = seq_ok(d, d->dh, false)) return e;
  if (pnn_status e = seq_ok(d, d->dx, true)) return e;
  if (pnn_status e = seq_ok(d, d->dgate, true)) return e;
  if (d->batch == 0 || d->channels == 0) return PNN_OK;
  if (d->length > 0 && (x == nullptr || gate == nullptr || states == nullptr || dh == nullptr || dx == nullptr ||
                        dgate == nullptr))
    return PNN_ERR_NULL;
  if (workspace == nullptr && scan_ws_bytes(*d) > 0) return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(x, es) || !aligned(gate, es) || !aligned(dh, es) || !aligned(dx, es) || !aligned(dgate, es) ||
      !aligned(lengths, 4) || !aligned(states, 4) || !aligned(dhT, 4) || !aligned(dh0, 4) || !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  if (d->length > 0 && (dx == dgate || dx == x || dx == gate || dx == dh || dgate == x || dgate == gate || dgate == dh))
    return PNN_ERR_SHAPE;
  ScanArgs a = {};
  a.x = x;
  a.gate = gate;
  a.lengths = lengths;
  a.states = const_cast<float*>(states);
  a.dh = dh;
  a.dhT = dhT;
  a.dx = dx;
  a.dgate = dgate;
  a.dh0 = dh0;
  a.ws = workspace;
  return launch_scan_bwd(*d, a, (hipStream_t)stream) ? PNN_ERR_HIP : PNN_OK;
}

pnn_status pnn_distill_fwd_bwd(const pnn_distill_desc* d, const void* logits, const int32_t* index,
                               const void* teacher, const int32_t* labels, const float* weight, float* loss,
                               void* dlogits, void* stream) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype) || !type_ok(d->teacher_dtype)) return PNN_ERR_DTYPE;
  if (d->rows < 0 || d->classes < 1 || d->top < 0) return PNN_ERR_SHAPE;
  if (d->rows > (1 << 28) || d->classes > MAX_COUNT || d->top > PNN_DISTILL_MAX_TOP) return PNN_ERR_TOO_LARGE;
  if (pnn_status e = rows_ok(d->rows, d->logit_stride, d->classes, false)) return e;
  if (pnn_status e = rows_ok(d->rows, d->top_stride, d->top, false)) return e;
  if (dlogits != nullptr)
    if (pnn_status e = rows_ok(d->rows, d->grad_stride, d->classes, true)) return e;
  const float tau = d->temperature;
  // the kernel's largest factor is log2(e) / tau
  if (!isfinite(tau) || !(tau > 0.0f) || !isfinite(1.44269504f / tau) || !isfinite(d->alpha * tau * tau) || !isfinite(d->scale))
    return PNN_ERR_VALUE;
  if (d->rows == 0) return PNN_OK;
  if (logits == nullptr || loss == nullptr || (d->top > 0 && (index == nullptr || teacher == nullptr)))
    return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(logits, es) || !aligned(dlogits, es) || !aligned(index, 4) ||
      !aligned(teacher, type_size(d->teacher_dtype)) || !aligned(labels, 4) || !aligned(weight, 4) || !aligned(loss, 4))
    return PNN_ERR_ALIGN;
  if (dlogits == logits && d->rows > 1 && d->grad_stride != d->logit_stride) return PNN_ERR_SHAPE;
  return launch_distill(*d, logits, index, teacher, labels, weight, loss, dlogits, (hipStream_t)stream) ? PNN_ERR_HIP
                                                                                                        : PNN_OK;
}

pnn_status pnn_linattn_sizes(const pnn_linattn_desc* d, size_t* forward, size_t* backward) {
  if (forward == nullptr || backward == nullptr) return PNN_ERR_NULL;
  if (pnn_status e = linattn_ok(d)) return e;
  *forward = (size_t)lin_fwd_bytes(*d);
  *backward = (size_t)lin_bwd(*d).bytes;
  return PNN_OK;
}

pnn_status pnn_linattn_fwd(const pnn_linattn_desc* d, const void* q, const void* k, const void* v,
                           const float* log_decay, const int32_t* lengths, const float* s0, void* o, float* sT,
                           void* workspace, void* stream) {
  if (pnn_status e = linattn_ok(d)) return e;
  if (pnn_status e = linattn_in_ok(d)) return e;
  if (pnn_status e = heads_ok(d, d->o, d->heads, d->value_width, true)) return e;
  if (d->batch == 0) return PNN_OK;
  if (log_decay == nullptr || (d->length > 0 && (q == nullptr || k == nullptr || v == nullptr || o == nullptr)) ||
      (workspace == nullptr && lin_fwd_bytes(*d) > 0))
    return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(o, es) || !aligned(log_decay, 4) ||
      !aligned(lengths, 4) || !aligned(s0, 4) || !aligned(sT, 4) || !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  if (d->length == 0) q = k = v = nullptr, o = nullptr;
  const void* const ws = lin_fwd_bytes(*d) > 0 ? workspace : nullptr;
  if (meet({o, sT}, {q, k, v, log_decay, lengths, ws}) || meet({o}, {s0})) return PNN_ERR_SHAPE;
  return launch_linattn_fwd(*d, q, k, v, log_decay, lengths, s0, o, sT, workspace, (hipStream_t)stream) ? PNN_ERR_HIP
                                                                                                        : PNN_OK;
}

pnn_status pnn_linattn_bwd(const pnn_linattn_desc* d, const void* q, const void* k, const void* v,
                           const float* log_decay, const int32_t* lengths, const float* s0, const void* dout,
                           const float* dsT, void* dq, void* dk, void* dv, float* ds0, void* workspace, void* stream) {
  if (pnn_status e = linattn_ok(d)) return e;
  if (pnn_status e = linattn_in_ok(d)) return e;
  if (pnn_status e = heads_ok(d, d->dout, d->heads, d->value_width, false)) return e;
  if (pnn_status e = heads_ok(d, d->dq, d->heads, d->key_width, true)) return e;
  if (pnn_status e = heads_ok(d, d->dk, d->kv_heads, d->key_width, true)) return e;
  if (pnn_status e = heads_ok(d, d->dv, d->kv_heads, d->value_width, true)) return e;
  if (lin_head_threads(*d) > (((int64_t)1 << 32) - 256)) return PNN_ERR_TOO_LARGE;
  if (d->batch == 0) return PNN_OK;
  if (log_decay == nullptr ||
      (d->length > 0 && (q == nullptr || k == nullptr || v == nullptr || dout == nullptr || dq == nullptr ||
                         dk == nullptr || dv == nullptr)) ||
      (workspace == nullptr && lin_bwd(*d).bytes > 0))
    return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(dout, es) || !aligned(dq, es) ||
      !aligned(dk, es) || !aligned(dv, es) || !aligned(log_decay, 4) || !aligned(lengths, 4) || !aligned(s0, 4) ||
      !aligned(dsT, 4) || !aligned(ds0, 4) || !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  if (d->length == 0) q = k = v = dout = nullptr, dq = dk = dv = nullptr;
  const void* const ws = lin_bwd(*d).bytes > 0 ? workspace : nullptr;
  if (meet({dq, dk, dv, ds0}, {q, k, v, dout, log_decay, lengths, s0, dsT, ws})) return PNN_ERR_SHAPE;
  return launch_linattn_bwd(*d, q, k, v, log_decay, lengths, s0, dout, dsT, dq, dk, dv, ds0, workspace,
                            (hipStream_t)stream)
             ? PNN_ERR_HIP
             : PNN_OK;
}

pnn_status pnn_norm_fwd(const pnn_norm_desc* d, const void* x, const float* w_post, const void* gate, const void* res,
                        const float* w_pre, void* h, void* y, void* stream) {
  if (pnn_status e = norm_ok(d)) return e;
  if (pnn_status e = norm_rows_ok(d, d->x, false)) return e;
  if (gate != nullptr)
    if (pnn_status e = norm_rows_ok(d, d->gate, false)) return e;
  if (res != nullptr)
    if (pnn_status e = norm_rows_ok(d, d->res, false)) return e;
  if (h != nullptr)
    if (pnn_status e = norm_rows_ok(d, d->h, true)) return e;
  if (d->pre)
    if (pnn_status e = norm_rows_ok(d, d->y, true)) return e;
  if (d->rows == 0) return PNN_OK;
  if (x == nullptr || (d->pre && y == nullptr) || (!d->pre && h == nullptr)) return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!d->pre) y = nullptr;
  if (!aligned(x, es) || !aligned(w_post, 4) || !aligned(gate, es) || !aligned(res, es) || !aligned(w_pre, 4) ||
      !aligned(h, es) || !aligned(y, es))
    return PNN_ERR_ALIGN;
  if (meet({h, y}, {x, gate, d->post ? w_post : nullptr, d->pre ? w_pre : nullptr}) || meet({y}, {res})) return PNN_ERR_SHAPE;
  if (h != nullptr && h == res && !same(d->h, d->res, d)) return PNN_ERR_SHAPE;
  return launch_norm_fwd(*d, x, w_post, gate, res, w_pre, h, y, (hipStream_t)stream) ? PNN_ERR_HIP : PNN_OK;
}

pnn_status pnn_norm_workspace_size(const pnn_norm_desc* d, size_t* bytes) {
  if (bytes == nullptr) return PNN_ERR_NULL;
  if (pnn_status e = norm_ok(d)) return e;
  *bytes = (size_t)norm_ws_bytes(*d);
  return PNN_OK;
}

pnn_status pnn_norm_bwd(const pnn_norm_desc* d, const void* x, const float* w_post, const void* gate, const void* res,
                        const float* w_pre, const void* dy, const void* dh, void* dx, void* dgate, void* dres,
                        float* dw_post, float* dw_pre, int accumulate, void* workspace, void* stream) {
  if (pnn_status e = norm_ok(d)) return e;
  if (!d->pre) res = dy = nullptr, dw_pre = nullptr;
  if (!d->post) dw_post = nullptr;
  if (gate == nullptr) dgate = nullptr;
  const bool stored = d->pre && d->stored, needs_x = d->post || (d->pre && !stored) || gate != nullptr;
  if (!needs_x) x = nullptr;
  const struct {
    const void* p;
    const pnn_row_stride& s;
    bool out;
  } tensors[8] = {{x, d->x, false},   {gate, d->gate, false}, {res, stored ? d->h : d->res, false}, {dy, d->dy, false},
                  {dh, d->dh, false}, {dx, d->dx, true},      {dgate, d->dgate, true}, {dres, d->dres, true}};
  for (const auto& t : tensors)
    if (t.p != nullptr)
      if (pnn_status e = norm_rows_ok(d, t.s, t.out)) return e;
  if (dx == nullptr && dgate == nullptr && dres == nullptr && dw_post == nullptr && dw_pre == nullptr) return PNN_OK;
  if (d->rows > 0 && ((needs_x && x == nullptr) || (d->pre && dy == nullptr) || (stored && res == nullptr)))
    return PNN_ERR_NULL;
  if (d->rows > 0 && (dw_post != nullptr || dw_pre != nullptr) && workspace == nullptr) return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  for (const auto& t : tensors)
    if (!aligned(t.p, es)) return PNN_ERR_ALIGN;
  if (!aligned(w_post, 4) || !aligned(w_pre, 4) || !aligned(dw_post, 4) || !aligned(dw_pre, 4) ||
      !aligned(workspace, 256))
    return PNN_ERR_ALIGN;
  const void* const ws = dw_post != nullptr || dw_pre != nullptr ? workspace : nullptr;
  if (meet({dx, dgate, dres, dw_post, dw_pre}, {x, gate, res, dy, w_post, w_pre, ws}) ||
      meet({dx, dgate, dw_post, dw_pre}, {dh}) || (dres != nullptr && dres == dh && !same(d->dres, d->dh, d)))
    return PNN_ERR_SHAPE;
  return launch_norm_bwd(*d, x, w_post, gate, res, w_pre, dy, dh, dx, dgate, dres, dw_post, dw_pre, accumulate, workspace,
                         (hipStream_t)stream)
             ? PNN_ERR_HIP
             : PNN_OK;
}

pnn_status pnn_policy_fwd_bwd(const pnn_policy_desc* d, const void* logits, const int32_t* tokens,
                              const float* advantage, const float* old, const float* ref, const float* weight,
                              float* loss, float* logp, void* dlogits, void* stream) {
  if (d == nullptr) return PNN_ERR_NULL;
  if (!type_ok(d->dtype)) return PNN_ERR_DTYPE;
  if (d->rows < 0 || d->classes < 1) return PNN_ERR_SHAPE;
  if (d->rows > (1 << 28) || d->classes > MAX_COUNT) return PNN_ERR_TOO_LARGE;
  if (pnn_status e = rows_ok(d->rows, d->logit_stride, d->classes, false)) return e;
  if (dlogits != nullptr)
    if (pnn_status e = rows_ok(d->rows, d->grad_stride, d->classes, true)) return e;
  const float tau = d->temperature;
  if (!isfinite(tau) || !(tau > 0.0f) || !isfinite(1.44269504f / tau) || !isfinite(d->clip_low) ||
      !isfinite(d->clip_high) || d->clip_low < 0.0f || d->clip_high < 0.0f || !isfinite(d->kl) || !isfinite(d->scale) ||
      !isfinite(d->scale / tau))
    return PNN_ERR_VALUE;
  if (d->rows == 0) return PNN_OK;
  if (logits == nullptr || tokens == nullptr || advantage == nullptr || loss == nullptr ||
      (d->kl != 0.0f && ref == nullptr))
    return PNN_ERR_NULL;
  const int es = type_size(d->dtype);
  if (!aligned(logits, es) || !aligned(dlogits, es) || !aligned(tokens, 4) || !aligned(advantage, 4) ||
      !aligned(old, 4) || !aligned(ref, 4) || !aligned(weight, 4) || !aligned(loss, 4) || !aligned(logp, 4))
    return PNN_ERR_ALIGN;
  if (dlogits == logits && d->rows > 1 && d->grad_stride != d->logit_stride) return PNN_ERR_SHAPE;
  if (meet({loss, logp, dlogits}, {tokens, advantage, old, ref, weight}) || meet({loss, logp}, {logits})) return PNN_ERR_SHAPE;
  return launch_policy(*d, logits, tokens, advantage, old, ref, weight, loss, logp, dlogits, (hipStream_t)stream)
             ? PNN_ERR_HIP
             : PNN_OK;
}

}  // extern "C"
