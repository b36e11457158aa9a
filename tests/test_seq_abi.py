"""Host-side checks of the sequence operators' C ABI (no GPU needed): exports, sizes and refusals.  Refused calls
enqueue nothing, so the pointers below are never dereferenced."""
import ctypes
import os
import re

import pytest

B = pytest.importorskip("paper_2103_08802_amd.binding")
from paper_2103_08802_amd import seq as Q  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pnn_seq.h")
P = 1 << 30            # some device address, 256-byte aligned
NULL, SHAPE, DTYPE, ALIGN, LARGE, VALUE = -1, -2, -3, -8, -9, -10


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libpnn.so not built")
    return Q.lib()


def test_header_declarations_are_exported(L):
    text = open(HEADER).read()
    declared = set(re.findall(r"^\s*pnn_status\s+(\w+)\s*\(", text, re.M))
    assert declared == set(Q.EXPORTS)
    for name in declared:
        assert hasattr(L, name), name
    assert int(re.search(r"PNN_DISTILL_MAX_TOP (\d+)", text).group(1)) == Q.DISTILL_MAX_TOP
    assert B.pnn_status_string(VALUE) == "a scalar argument is out of its range"


def _embed(**kw):
    return Q.EmbedDesc(**{**dict(dtype=1, table_dtype=1, token_bytes=8, n=100, vocab=50, width=16, table_stride=16,
                                 row_stride=16, scale=1.0), **kw})


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=2), DTYPE), (dict(table_dtype=-1), DTYPE), (dict(token_bytes=2), DTYPE),
    (dict(n=-1), SHAPE), (dict(vocab=-1), SHAPE), (dict(width=-1), SHAPE),
    (dict(row_stride=-16), SHAPE), (dict(table_stride=-1), SHAPE),
    (dict(n=(1 << 28) + 1), LARGE), (dict(vocab=(1 << 31) - 1), LARGE), (dict(width=(1 << 23) + 1), LARGE),
    (dict(row_stride=1 << 60), LARGE), (dict(vocab=1 << 30, table_stride=1 << 31), LARGE),
    (dict(scale=float("nan")), VALUE), (dict(scale=float("inf")), VALUE)])
def test_embed_descriptions(L, kw, st):
    d = _embed(**kw)
    size = ctypes.c_size_t()
    assert L.pnn_embed_workspace_size(d, ctypes.byref(size)) == st
    assert L.pnn_embed_fwd(d, P, P, P + 256, None) == st
    assert L.pnn_embed_bwd(d, P, P, P + 256, 0, P, None) == st


def test_embed_arguments(L):
    d = _embed()
    size = ctypes.c_size_t()
    assert L.pnn_embed_workspace_size(None, ctypes.byref(size)) == NULL
    assert L.pnn_embed_workspace_size(d, None) == NULL
    assert L.pnn_embed_workspace_size(d, ctypes.byref(size)) == 0 and size.value % 256 == 0
    for args, st in (((None, P, P + 64), NULL), ((P, None, P + 64), NULL), ((P, P, None), NULL),
                     ((P + 1, P, P + 64), ALIGN), ((P, P + 4, P + 64), ALIGN), ((P, P, P + 65), ALIGN),
                     ((P, P, P), SHAPE)):
        assert L.pnn_embed_fwd(d, *args, None) == st, args
    assert L.pnn_embed_fwd(None, P, P, P, None) == NULL
    assert L.pnn_embed_fwd(_embed(row_stride=15), P, P, P + 64, None) == SHAPE       # output rows overlap
    for args, st in (((None, P, P + 64, 0, P), NULL), ((P, None, P + 64, 0, P), NULL), ((P, P, None, 0, P), NULL),
                     ((P, P, P + 64, 0, None), NULL), ((P + 1, P, P + 64, 0, P), ALIGN),
                     ((P, P + 4, P + 64, 0, P), ALIGN), ((P, P, P + 66, 0, P), ALIGN),
                     ((P, P, P + 64, 1, P + 128), ALIGN), ((P, P, P, 0, P), SHAPE)):
        assert L.pnn_embed_bwd(d, *args, None) == st, args
    assert L.pnn_embed_bwd(_embed(table_stride=15), P, P, P + 64, 0, P, None) == SHAPE
    assert L.pnn_embed_fwd(_embed(n=0), None, None, None, None) == 0                 # nothing to do
    assert L.pnn_embed_bwd(_embed(vocab=0, n=0), None, None, None, 0, None, None) == 0


def _scan(**kw):
    st = Q.SeqStride(10 * 16, 16)
    return Q.ScanDesc(**{**dict(dtype=1, batch=3, length=10, channels=16, x=st, gate=st, h=st, dh=st, dx=st,
                                dgate=st), **kw})


FWD = dict(x=P, gate=P + 4096, lengths=None, h0=None, h=P + 8192, hT=None, states=None, ws=P)
BWD = dict(x=P, gate=P + 4096, lengths=None, states=P + 64, dh=P + 8192, dhT=None, dx=P + 16384, dgate=P + 20480,
           dh0=None, ws=P)


def _fwd(L, d, **kw):
    return L.pnn_scan_fwd(d, *{**FWD, **kw}.values(), None)


def _bwd(L, d, **kw):
    return L.pnn_scan_bwd(d, *{**BWD, **kw}.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=9), DTYPE), (dict(batch=-1), SHAPE), (dict(length=-1), SHAPE), (dict(channels=-2), SHAPE),
    (dict(x=Q.SeqStride(-160, 16)), SHAPE), (dict(gate=Q.SeqStride(160, -16)), SHAPE),
    (dict(x=Q.SeqStride(1 << 60, 16)), LARGE), (dict(gate=Q.SeqStride(16, 1 << 58)), LARGE),
    (dict(batch=1 << 31), LARGE), (dict(length=1 << 31), LARGE), (dict(channels=1 << 30, batch=2), LARGE)])
def test_scan_descriptions(L, kw, st):
    d = _scan(**kw)
    assert _fwd(L, d) == st and _bwd(L, d) == st


def test_scan_arguments(L):
    d = _scan()
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert L.pnn_scan_sizes(None, ctypes.byref(a), ctypes.byref(b)) == NULL
    assert L.pnn_scan_sizes(d, None, ctypes.byref(b)) == NULL
    assert L.pnn_scan_sizes(d, ctypes.byref(a), ctypes.byref(b)) == 0 and a.value >= 3 * 16 * 4
    assert _fwd(L, None) == NULL and _bwd(L, None) == NULL
    for k in ("x", "gate", "h"):
        assert _fwd(L, d, **{k: None}) == NULL
        assert _fwd(L, d, **{k: FWD[k] + 1}) == ALIGN
    for k in ("lengths", "h0", "hT", "states"):
        assert _fwd(L, d, **{k: P + 2}) == ALIGN
    assert _fwd(L, d, ws=P + 16) == ALIGN
    assert _fwd(L, d, h=FWD["x"]) == SHAPE and _fwd(L, d, h=FWD["gate"]) == SHAPE
    for k in ("x", "gate", "states", "dh", "dx", "dgate"):
        assert _bwd(L, d, **{k: None}) == NULL
        assert _bwd(L, d, **{k: BWD[k] + 1}) == ALIGN
    for k in ("lengths", "dhT", "dh0"):
        assert _bwd(L, d, **{k: P + 2}) == ALIGN
    assert _bwd(L, d, ws=P + 16) == ALIGN
    for k in ("x", "gate", "dh", "dgate"):
        assert _bwd(L, d, dx=BWD[k]) == SHAPE
    for k in ("x", "gate", "dh"):
        assert _bwd(L, d, dgate=BWD[k]) == SHAPE
    # outputs whose rows meet: steps, sequences, and both interleaved
    for s in (Q.SeqStride(160, 15), Q.SeqStride(15, 160), Q.SeqStride(100, 16), Q.SeqStride(16, 40), Q.SeqStride(0, 0)):
        assert _fwd(L, _scan(h=s)) == SHAPE
        assert _bwd(L, _scan(dx=s)) == SHAPE and _bwd(L, _scan(dgate=s)) == SHAPE
    assert _fwd(L, _scan(batch=0), x=None, gate=None, h=None) == 0
    assert _bwd(L, _scan(channels=0), x=None) == 0


def _distill(**kw):
    return Q.DistillDesc(**{**dict(dtype=1, teacher_dtype=0, rows=4, classes=32, top=8, logit_stride=32,
                                   grad_stride=32, top_stride=8, temperature=2.0, alpha=0.5, scale=1.0), **kw})


DIS = dict(z=P, index=P + 4096, teacher=P + 8192, labels=None, weight=None, loss=P + 12288, dz=P + 16384)


def _dis(L, d, **kw):
    return L.pnn_distill_fwd_bwd(d, *{**DIS, **kw}.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=3), DTYPE), (dict(teacher_dtype=3), DTYPE), (dict(rows=-1), SHAPE), (dict(classes=0), SHAPE),
    (dict(top=-1), SHAPE), (dict(logit_stride=-1), SHAPE), (dict(top_stride=-8), SHAPE), (dict(grad_stride=31), SHAPE),
    (dict(top=Q.DISTILL_MAX_TOP + 1), LARGE), (dict(rows=(1 << 28) + 1), LARGE), (dict(classes=1 << 31), LARGE),
    (dict(logit_stride=1 << 60), LARGE), (dict(temperature=0.0), VALUE), (dict(temperature=-1.0), VALUE),
    (dict(temperature=float("nan")), VALUE), (dict(temperature=float("inf")), VALUE), (dict(temperature=1e-40), VALUE),
    (dict(temperature=1e30), VALUE), (dict(alpha=float("nan")), VALUE), (dict(scale=float("inf")), VALUE)])
def test_distill_descriptions(L, kw, st):
    assert _dis(L, _distill(**kw)) == st


def test_distill_arguments(L):
    d = _distill()
    assert _dis(L, None) == NULL
    for k in ("z", "index", "teacher", "loss"):
        assert _dis(L, d, **{k: None}) == NULL
    for k in ("z", "index", "teacher", "loss", "dz"):
        assert _dis(L, d, **{k: DIS[k] + 1}) == ALIGN
    for k in ("labels", "weight"):
        assert _dis(L, d, **{k: P + 2}) == ALIGN
    assert _dis(L, _distill(grad_stride=40), dz=DIS["z"]) == SHAPE
    assert _dis(L, _distill(rows=0), z=None, loss=None) == 0


def test_python_descriptions():
    import torch
    t = torch.zeros(6, 8)
    tok = torch.zeros(6, dtype=torch.int64)
    with pytest.raises(ValueError):
        Q.embed_desc(t, tok[:5], t)
    with pytest.raises(ValueError):
        Q.embed_desc(t.t(), tok[:6], t)
    with pytest.raises(TypeError):
        Q.embed_desc(t, tok.to(torch.int16), t)
    with pytest.raises(TypeError):
        Q.embed_desc(t.half(), tok, t.half())
    x = torch.zeros(2, 5, 4)
    with pytest.raises(ValueError):
        Q.scan_desc(x, x[:, :4], x)
    with pytest.raises(ValueError):
        Q.scan_desc(x, x, x.bfloat16())
    with pytest.raises(ValueError):
        Q.scan_desc(x, x, torch.zeros(2, 4, 5).transpose(1, 2))
    with pytest.raises(ValueError):
        Q.distill_desc(t, t[:5])
    with pytest.raises(ValueError):
        Q.distill_desc(t, t, t.bfloat16())
    both = torch.zeros(2, 5, 8)
    d = Q.scan_desc(both[..., :4], both[..., 4:], x)
    assert (d.x.batch, d.x.step, d.gate.step, d.h.step, d.channels) == (40, 8, 8, 4, 4)
