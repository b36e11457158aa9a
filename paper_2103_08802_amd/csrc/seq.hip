// Entry points of the sequence operators (pnn_seq.h): argument checks, then the launchers.
#include <math.h>

#include "pnn_seq.h"
#include "seq_internal.h"

using namespace pnn;

namespace {

constexpr int64_t MAX_COUNT = 0x7fffffff;
constexpr int64_t MAX_SPAN = int64_t(1) << 60;

bool type_ok(int t) { return t == PNN_F32 || t == PNN_BF16; }
int type_size(int t) { return t == PNN_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

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

}  // extern "C"
