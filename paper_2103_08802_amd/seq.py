"""Thin ctypes binding of libpnn's sequence operators (``include/pnn_seq.h``): token embedding, gated linear
recurrence, linear attention, norms, distillation and policy loss.

Every ``pnn_*`` function has the name of the C entry point it calls and takes a description, device
pointers as Python ints or objects with ``data_ptr()`` (None: NULL) and a stream.  ``embed_desc``,
``scan_desc``, ``distill_desc``, ``linattn_desc``, ``norm_desc`` and ``policy_desc`` fill the descriptions from
tensors; fill one once and use it for every call on tensors of the same types, shapes and strides.  As in
``binding``, nothing falls back to anything else: a refused call raises ``PnnError``.
"""
from __future__ import annotations

import ctypes
import weakref

from . import binding
from .binding import PNN_BF16, PNN_F32, PnnError  # noqa: F401

# every symbol include/pnn_seq.h declares
EXPORTS = ["pnn_embed_fwd", "pnn_embed_workspace_size", "pnn_embed_bwd", "pnn_scan_sizes", "pnn_scan_fwd",
           "pnn_scan_bwd", "pnn_distill_fwd_bwd", "pnn_linattn_sizes", "pnn_linattn_fwd", "pnn_linattn_bwd",
           "pnn_norm_fwd", "pnn_norm_workspace_size", "pnn_norm_bwd", "pnn_policy_fwd_bwd"]
DISTILL_MAX_TOP = 1024
LINATTN_MAX_WIDTH = 256
NORM_MAX_WIDTH = 16384

_i, _i64, _f, _vp = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class EmbedDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("table_dtype", _i), ("token_bytes", _i), ("n", _i64), ("vocab", _i64),
                ("width", _i64), ("table_stride", _i64), ("row_stride", _i64), ("scale", _f)]


class SeqStride(ctypes.Structure):
    _fields_ = [("batch", _i64), ("step", _i64)]


class ScanDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("batch", _i64), ("length", _i64), ("channels", _i64)] + \
               [(n, SeqStride) for n in ("x", "gate", "h", "dh", "dx", "dgate")]


class DistillDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("teacher_dtype", _i), ("rows", _i64), ("classes", _i64), ("top", _i64),
                ("logit_stride", _i64), ("grad_stride", _i64), ("top_stride", _i64), ("temperature", _f),
                ("alpha", _f), ("scale", _f)]


class HeadStride(ctypes.Structure):
    _fields_ = [("batch", _i64), ("step", _i64), ("head", _i64)]


class LinattnDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("batch", _i64), ("length", _i64), ("heads", _i64), ("kv_heads", _i64),
                ("key_width", _i64), ("value_width", _i64)] + \
               [(n, HeadStride) for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")] + [("scale", _f)]


class RowStride(ctypes.Structure):
    _fields_ = [("row", _i64), ("head", _i64)]


class NormDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("rows", _i64), ("heads", _i64), ("width", _i64), ("post", _i), ("pre", _i)] + \
               [(n, RowStride) for n in ("x", "gate", "res", "h", "y", "dy", "dh", "dx", "dgate", "dres")] + \
               [("eps", _f), ("alpha", _f), ("stored", _i)]
    sum = kept = None        # norm_desc: what pnn_norm_bwd knows the described h by, and (the residual it takes instead)


class PolicyDesc(ctypes.Structure):
    _fields_ = [("dtype", _i), ("rows", _i64), ("classes", _i64), ("logit_stride", _i64), ("grad_stride", _i64),
                ("temperature", _f), ("clip_low", _f), ("clip_high", _f), ("kl", _f), ("scale", _f)]


_lib = None


def lib():
    """libpnn.so with the argument types of the sequence operators set."""
    global _lib
    if _lib is not None:
        return _lib
    L = binding.lib()
    szp = ctypes.POINTER(ctypes.c_size_t)
    E, S, D = ctypes.POINTER(EmbedDesc), ctypes.POINTER(ScanDesc), ctypes.POINTER(DistillDesc)
    L.pnn_embed_fwd.argtypes = [E] + [_vp] * 4
    L.pnn_embed_workspace_size.argtypes = [E, szp]
    L.pnn_embed_bwd.argtypes = [E, _vp, _vp, _vp, _i, _vp, _vp]
    L.pnn_scan_sizes.argtypes = [S, szp, szp]
    L.pnn_scan_fwd.argtypes = [S] + [_vp] * 9
    L.pnn_scan_bwd.argtypes = [S] + [_vp] * 11
    L.pnn_distill_fwd_bwd.argtypes = [D] + [_vp] * 8
    A = ctypes.POINTER(LinattnDesc)
    L.pnn_linattn_sizes.argtypes = [A, szp, szp]
    L.pnn_linattn_fwd.argtypes = [A] + [_vp] * 10
    L.pnn_linattn_bwd.argtypes = [A] + [_vp] * 14
    N = ctypes.POINTER(NormDesc)
    L.pnn_norm_fwd.argtypes = [N] + [_vp] * 8
    L.pnn_norm_workspace_size.argtypes = [N, szp]
    L.pnn_norm_bwd.argtypes = [N] + [_vp] * 12 + [_i, _vp, _vp]
    L.pnn_policy_fwd_bwd.argtypes = [ctypes.POINTER(PolicyDesc)] + [_vp] * 10
    _lib = L
    return L


_ptr, _check = binding._ptr, binding._check


# ------------------------------------------------------------------------------------------------
# descriptions from tensors
# ------------------------------------------------------------------------------------------------

def _dtype(t):
    name = str(t.dtype)
    if name not in ("torch.float32", "torch.bfloat16"):
        raise TypeError(f"float32 or bfloat16 expected, not {t.dtype}")
    return PNN_F32 if name == "torch.float32" else PNN_BF16


def _rows(t, what):
    """(rows, width, elements from row to row) of a matrix with contiguous rows."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a matrix with contiguous rows expected, not shape {tuple(t.shape)}, "
                         f"strides {tuple(t.stride())}")
    return t.shape[0], t.shape[1], t.stride(0) if t.shape[0] > 1 else t.shape[1]


def embed_desc(table, tokens, rows, scale=1.0):
    """Table [vocab][width] (or its gradient), tokens (any shape, contiguous, int32 or int64) and the rows
    [n][width] that belong to them (``out`` or ``dout``)."""
    vocab, width, ts = _rows(table, "table")
    n, w, rs = _rows(rows, "rows")
    if w != width or n != tokens.numel():
        raise ValueError(f"table {tuple(table.shape)}, {tokens.numel()} tokens and rows {tuple(rows.shape)} differ")
    if not tokens.is_contiguous() or str(tokens.dtype) not in ("torch.int32", "torch.int64"):
        raise TypeError("tokens: contiguous int32 or int64 expected")
    return EmbedDesc(_dtype(rows), _dtype(table), tokens.element_size(), n, vocab, width, ts, rs, scale)


def _seq_stride(t, shape, dtype, what):
    if tuple(t.shape) != shape or _dtype(t) != dtype or (shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, {t.dtype}, strides {tuple(t.stride())} do not fit")
    return SeqStride(t.stride(0), t.stride(1))


def scan_desc(x, gate, h, dh=None, dx=None, dgate=None):
    """Tensors [batch][length][channels] with contiguous channels, all of one type; the gradients' may be left
    out for a description that only the forward uses."""
    if x.dim() != 3:
        raise ValueError(f"x: [batch][length][channels] expected, not {tuple(x.shape)}")
    shape, dt = tuple(x.shape), _dtype(x)
    st = [SeqStride(0, 0) if t is None else _seq_stride(t, shape, dt, n)
          for n, t in (("x", x), ("gate", gate), ("h", h), ("dh", dh), ("dx", dx), ("dgate", dgate))]
    return ScanDesc(dt, *shape, *st)


def distill_desc(logits, teacher, dlogits=None, temperature=1.0, alpha=1.0, scale=1.0):
    """Logits [rows][classes], the teacher's logits [rows][top] (their index tensor has the same shape and
    strides) and, unless only the loss is wanted, dlogits like logits."""
    rows, classes, ls = _rows(logits, "logits")
    n, top, ks = _rows(teacher, "teacher")
    gs = ls
    if dlogits is not None:
        gn, gw, gs = _rows(dlogits, "dlogits")
        if (gn, gw) != (rows, classes) or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits and logits differ in shape or type")
    if n != rows:
        raise ValueError(f"{n} rows of the teacher, {rows} of logits")
    return DistillDesc(_dtype(logits), _dtype(teacher), rows, classes, top, ls, gs, ks, temperature, alpha, scale)


def _head_stride(t, shape, dtype, what):
    if tuple(t.shape) != shape or _dtype(t) != dtype or (shape[3] > 1 and t.stride(3) != 1):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, {t.dtype}, strides {tuple(t.stride())} do not fit "
                         f"[batch][length][heads][width] {shape}")
    return HeadStride(t.stride(0), t.stride(1), t.stride(2))


def linattn_desc(q, k, v, o, dout=None, dq=None, dk=None, dv=None, scale=1.0):
    """Queries [batch][length][heads][key width], keys and values [batch][length][kv heads][..], outputs
    [batch][length][heads][value width], each with contiguous widths, all of one type; the gradients' (shaped like o, q,
    k, v) may be left out for a description that only the forward uses."""
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v: [batch][length][heads][width] expected")
    dt = _dtype(q)
    B, T, H, K = q.shape
    kv, V = k.shape[2], v.shape[3]
    qs, ks, vs, os = (B, T, H, K), (B, T, kv, K), (B, T, kv, V), (B, T, H, V)
    st = [HeadStride(0, 0, 0) if t is None else _head_stride(t, shape, dt, n)
          for n, t, shape in (("q", q, qs), ("k", k, ks), ("v", v, vs), ("o", o, os), ("dout", dout, os), ("dq", dq, qs),
                              ("dk", dk, ks), ("dv", dv, vs))]
    return LinattnDesc(dt, B, T, H, kv, K, V, *st, scale)


def norm_desc(x, gate=None, res=None, h=None, y=None, dy=None, dh=None, dx=None, dgate=None, dres=None, post=False,
              pre=False, eps=1e-5, alpha=1.0, stored=None, kept=False):
    """Tensors [rows][heads][width], or [rows][width] for one head, with contiguous widths, all of x's type and shape; those
    that no call uses may be left out.  ``post``: norm of x, ``pre``: norm of h.

    ``stored``: whether the ``res`` that pnn_norm_bwd gets is h as the forward stored it (True; the form after a forward in
    place) or the residual (False).  Left out it is the residual, and the call refuses the tensor described as h, which
    may be either.  ``kept``: what h is the sum of stays as it is until the backward, which, given the tensor
    described as h, forms it again from x, gate and the tensor described as res, without its rounding; such a description
    holds that tensor and serves its own tensors only."""
    if x.dim() not in (2, 3):
        raise ValueError(f"x: [rows][heads][width] or [rows][width] expected, not {tuple(x.shape)}")
    if kept and (stored or h is None or (res is not None and res.data_ptr() == h.data_ptr() != 0)):
        raise ValueError("kept: h, apart from res, and a sum that the backward forms again")
    dt, shape = _dtype(x), tuple(x.shape)
    st = []
    for n, t in (("x", x), ("gate", gate), ("res", res), ("h", h), ("y", y), ("dy", dy), ("dh", dh), ("dx", dx),
                 ("dgate", dgate), ("dres", dres)):
        if t is None:
            st.append(RowStride(0, 0))
            continue
        if tuple(t.shape) != shape or _dtype(t) != dt or (shape[-1] > 1 and t.stride(-1) != 1):
            raise ValueError(f"{n}: shape {tuple(t.shape)}, {t.dtype}, strides {tuple(t.stride())} do not fit")
        st.append(RowStride(t.stride(0), t.stride(1) if len(shape) == 3 else shape[-1]))
    d = NormDesc(dt, shape[0], shape[1] if len(shape) == 3 else 1, shape[-1], int(bool(post)), int(bool(pre)), *st,
                 eps, alpha, int(bool(stored)))
    if kept or (stored is None and h is not None):
        d.sum = weakref.ref(h)
    if kept:
        d.kept = (res,)
    return d


def policy_desc(logits, dlogits=None, temperature=1.0, clip_low=0.2, clip_high=0.2, kl=0.0, scale=1.0):
    """Logits [rows][classes] and, unless only the loss and the log probabilities are wanted, dlogits like logits."""
    rows, classes, ls = _rows(logits, "logits")
    gs = ls
    if dlogits is not None:
        gn, gw, gs = _rows(dlogits, "dlogits")
        if (gn, gw) != (rows, classes) or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits and logits differ in shape or type")
    return PolicyDesc(_dtype(logits), rows, classes, ls, gs, temperature, clip_low, clip_high, kl, scale)


# ------------------------------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ------------------------------------------------------------------------------------------------

def pnn_embed_fwd(desc, table, tokens, out, stream):
    _check(lib().pnn_embed_fwd(desc, _ptr(table), _ptr(tokens), _ptr(out), stream), "pnn_embed_fwd")


def pnn_embed_workspace_size(desc):
    v = ctypes.c_size_t()
    _check(lib().pnn_embed_workspace_size(desc, ctypes.byref(v)), "pnn_embed_workspace_size")
    return v.value


def pnn_embed_bwd(desc, dout, tokens, dtable, accumulate, workspace, stream):
    _check(lib().pnn_embed_bwd(desc, _ptr(dout), _ptr(tokens), _ptr(dtable), int(bool(accumulate)),
                               _ptr(workspace), stream), "pnn_embed_bwd")


def pnn_scan_sizes(desc):
    """(bytes of ``states``, bytes of the workspace)"""
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().pnn_scan_sizes(desc, ctypes.byref(a), ctypes.byref(b)), "pnn_scan_sizes")
    return a.value, b.value


def pnn_scan_fwd(desc, x, gate, lengths, h0, h, hT, states, workspace, stream):
    _check(lib().pnn_scan_fwd(desc, _ptr(x), _ptr(gate), _ptr(lengths), _ptr(h0), _ptr(h), _ptr(hT),
                              _ptr(states), _ptr(workspace), stream), "pnn_scan_fwd")


def pnn_scan_bwd(desc, x, gate, lengths, states, dh, dhT, dx, dgate, dh0, workspace, stream):
    _check(lib().pnn_scan_bwd(desc, _ptr(x), _ptr(gate), _ptr(lengths), _ptr(states), _ptr(dh), _ptr(dhT),
                              _ptr(dx), _ptr(dgate), _ptr(dh0), _ptr(workspace), stream), "pnn_scan_bwd")


def pnn_distill_fwd_bwd(desc, logits, index, teacher, labels, weight, loss, dlogits, stream):
    _check(lib().pnn_distill_fwd_bwd(desc, _ptr(logits), _ptr(index), _ptr(teacher), _ptr(labels), _ptr(weight),
                                     _ptr(loss), _ptr(dlogits), stream), "pnn_distill_fwd_bwd")


def pnn_linattn_sizes(desc):
    """Bytes of workspace: (forward, backward)"""
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().pnn_linattn_sizes(desc, ctypes.byref(a), ctypes.byref(b)), "pnn_linattn_sizes")
    return a.value, b.value


def pnn_linattn_fwd(desc, q, k, v, log_decay, lengths, s0, o, sT, workspace, stream):
    _check(lib().pnn_linattn_fwd(desc, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(lengths), _ptr(s0), _ptr(o),
                                 _ptr(sT), _ptr(workspace), stream), "pnn_linattn_fwd")


def pnn_linattn_bwd(desc, q, k, v, log_decay, lengths, s0, dout, dsT, dq, dk, dv, ds0, workspace, stream):
    _check(lib().pnn_linattn_bwd(desc, _ptr(q), _ptr(k), _ptr(v), _ptr(log_decay), _ptr(lengths), _ptr(s0), _ptr(dout),
                                 _ptr(dsT), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(ds0), _ptr(workspace), stream),
           "pnn_linattn_bwd")


def pnn_norm_fwd(desc, x, w_post, gate, res, w_pre, h, y, stream):
    _check(lib().pnn_norm_fwd(desc, _ptr(x), _ptr(w_post), _ptr(gate), _ptr(res), _ptr(w_pre), _ptr(h), _ptr(y), stream),
           "pnn_norm_fwd")


def pnn_norm_workspace_size(desc):
    v = ctypes.c_size_t()
    _check(lib().pnn_norm_workspace_size(desc, ctypes.byref(v)), "pnn_norm_workspace_size")
    return v.value


def _norm_sum(desc, res):
    """What stands in res's place in the backward: the residual or, if the description says so, h."""
    if desc.sum is None or res is None or not desc.pre:
        return res
    h, at = desc.sum(), _ptr(res)
    is_h = h is not None and at == h.data_ptr() != 0
    if desc.kept is None:
        if is_h:
            raise ValueError("res is the tensor described as h: norm_desc's stored says whether it is the sum here")
        return res
    if not is_h and at != _ptr(desc.kept[0]):
        raise ValueError("res: a description with kept serves its own tensors only")
    return desc.kept[0]


def pnn_norm_bwd(desc, x, w_post, gate, res, w_pre, dy, dh, dx, dgate, dres, dw_post, dw_pre, accumulate, workspace, stream):
    """``res``: the residual, or h (norm_desc's ``stored`` and ``kept``)."""
    res = _norm_sum(desc, res)
    _check(lib().pnn_norm_bwd(desc, _ptr(x), _ptr(w_post), _ptr(gate), _ptr(res), _ptr(w_pre), _ptr(dy), _ptr(dh), _ptr(dx),
                              _ptr(dgate), _ptr(dres), _ptr(dw_post), _ptr(dw_pre), int(bool(accumulate)),
                              _ptr(workspace), stream), "pnn_norm_bwd")


def pnn_policy_fwd_bwd(desc, logits, tokens, advantage, old, ref, weight, loss, logp, dlogits, stream):
    _check(lib().pnn_policy_fwd_bwd(desc, _ptr(logits), _ptr(tokens), _ptr(advantage), _ptr(old), _ptr(ref),
                                    _ptr(weight), _ptr(loss), _ptr(logp), _ptr(dlogits), stream), "pnn_policy_fwd_bwd")
