"""Thin ctypes binding of libpnn's sequence operators (``include/pnn_seq.h``): token embedding, gated linear
recurrence and distillation loss.

Every ``pnn_*`` function has the name of the C entry point it calls and takes a description, device
pointers as Python ints or objects with ``data_ptr()`` (None: NULL) and a stream.  ``embed_desc``,
``scan_desc`` and ``distill_desc`` fill the descriptions from tensors; fill one once and use it for every
call on tensors of the same types, shapes and strides.  As in ``binding``, nothing falls back to anything
else: a refused call raises ``PnnError``.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import PNN_BF16, PNN_F32, PnnError  # noqa: F401

# every symbol include/pnn_seq.h declares
EXPORTS = ["pnn_embed_fwd", "pnn_embed_workspace_size", "pnn_embed_bwd", "pnn_scan_sizes", "pnn_scan_fwd",
           "pnn_scan_bwd", "pnn_distill_fwd_bwd"]
DISTILL_MAX_TOP = 1024

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
