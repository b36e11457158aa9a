"""Host-side checks of linear attention, norms and the policy loss at the C ABI (no GPU needed): sizes and refusals.
Refused calls enqueue nothing, so the pointers below are never dereferenced."""
import ctypes
import os
import re

import pytest

B = pytest.importorskip("paper_2103_08802_amd.binding")
from paper_2103_08802_amd import seq as Q  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pnn_seq.h")
P = 1 << 30            # some device address, 256-byte aligned
NULL, SHAPE, DTYPE, ALIGN, LARGE, VALUE = -1, -2, -3, -8, -9, -10
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libpnn.so not built")
    return Q.lib()


def test_limits():
    text = open(HEADER).read()
    for name, value in (("PNN_LINATTN_MAX_WIDTH", Q.LINATTN_MAX_WIDTH), ("PNN_NORM_MAX_WIDTH", Q.NORM_MAX_WIDTH)):
        assert int(re.search(name + r" (\d+)", text).group(1)) == value


# ---- linear attention --------------------------------------------------------------------------

def _lin(**kw):
    q, k, v = Q.HeadStride(10 * 64, 64, 16), Q.HeadStride(10 * 32, 32, 16), Q.HeadStride(10 * 48, 48, 24)
    o = Q.HeadStride(10 * 96, 96, 24)
    return Q.LinattnDesc(**{**dict(dtype=1, batch=3, length=10, heads=4, kv_heads=2, key_width=16, value_width=24, q=q, k=k,
                                   v=v, o=o, dout=o, dq=q, dk=k, dv=v, scale=0.25), **kw})


S = 1 << 16
LFWD = dict(q=P, k=P + S, v=P + 2 * S, log_decay=P + 64, lengths=None, s0=None, o=P + 3 * S, sT=None, ws=P)
LBWD = dict(q=P, k=P + S, v=P + 2 * S, log_decay=P + 64, lengths=None, s0=None, dout=P + 3 * S, dsT=None, dq=P + 4 * S,
            dk=P + 5 * S, dv=P + 6 * S, ds0=None, ws=P)


def _lf(L, d, **kw):
    return L.pnn_linattn_fwd(d, *{**LFWD, **kw}.values(), None)


def _lb(L, d, **kw):
    return L.pnn_linattn_bwd(d, *{**LBWD, **kw}.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=2), DTYPE), (dict(batch=-1), SHAPE), (dict(length=-1), SHAPE), (dict(heads=0), SHAPE),
    (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(kv_heads=8), SHAPE), (dict(key_width=0), SHAPE),
    (dict(value_width=0), SHAPE), (dict(key_width=257), LARGE), (dict(value_width=257), LARGE),
    (dict(length=(1 << 30) + 1), LARGE), (dict(batch=1 << 21), LARGE), (dict(heads=1 << 21, kv_heads=1), LARGE),
    (dict(batch=1 << 15, heads=1 << 6), LARGE), (dict(length=1 << 28), LARGE), (dict(scale=NAN), VALUE),
    (dict(scale=INF), VALUE)])
def test_linattn_descriptions(L, kw, st):
    d = _lin(**kw)
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert L.pnn_linattn_sizes(d, ctypes.byref(a), ctypes.byref(b)) == st
    assert _lf(L, d) == st and _lb(L, d) == st


@pytest.mark.parametrize("which", ["q", "k", "v", "o", "dout", "dq", "dk", "dv"])
def test_linattn_strides(L, which):
    forward, backward = which in "qkvo", which != "o"
    out = which in ("o", "dq", "dk", "dv")
    width = 16 if which in ("q", "k", "dq", "dk") else 24
    for s, st in ((Q.HeadStride(-640, 64, 32), SHAPE), (Q.HeadStride(960, -96, 32), SHAPE), (Q.HeadStride(960, 96, -1), SHAPE),
                  (Q.HeadStride(1 << 60, 96, 24), LARGE), (Q.HeadStride(960, 1 << 58, 24), LARGE),
                  (Q.HeadStride(960, 96, 1 << 60), LARGE)):
        if forward:
            assert _lf(L, _lin(**{which: s})) == st, s
        if backward:
            assert _lb(L, _lin(**{which: s})) == st, s
    if out:                                          # rows that meet, whichever way round the dimensions are
        for s in (Q.HeadStride(960, 96, width - 1), Q.HeadStride(960, width - 1, 240), Q.HeadStride(width - 1, 96, 960),
                  Q.HeadStride(0, 0, 0), Q.HeadStride(100, 96, 24), Q.HeadStride(96, 24, 100)):
            assert (_lf if forward else _lb)(L, _lin(**{which: s})) == SHAPE, s


def test_linattn_arguments(L):
    d = _lin()
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert L.pnn_linattn_sizes(None, ctypes.byref(a), ctypes.byref(b)) == NULL
    assert L.pnn_linattn_sizes(d, None, ctypes.byref(b)) == NULL
    assert L.pnn_linattn_sizes(d, ctypes.byref(a), None) == NULL
    assert L.pnn_linattn_sizes(d, ctypes.byref(a), ctypes.byref(b)) == 0 and a.value == 0 and b.value % 256 == 0
    assert b.value >= 3 * 10 * 4 * (16 + 24) * 4         # single heads' gradients of shared keys and values
    long = _lin(length=1000, kv_heads=4, **{n: Q.HeadStride(1 << 20, 1 << 10, 24) for n in ("q", "k", "v", "o", "dout",
                                                                                           "dq", "dk", "dv")})
    assert L.pnn_linattn_sizes(long, ctypes.byref(a), ctypes.byref(b)) == 0 and a.value > 0 and b.value > 0
    assert _lf(L, long, ws=None) == NULL and _lb(L, long, ws=None) == NULL and _lb(L, d, ws=None) == NULL
    assert _lf(L, None) == NULL and _lb(L, None) == NULL
    for k in ("q", "k", "v", "o", "log_decay"):
        assert _lf(L, d, **{k: None}) == NULL
        assert _lf(L, d, **{k: LFWD[k] + 1}) == ALIGN
    for k in ("lengths", "s0", "sT"):
        assert _lf(L, d, **{k: P + 2}) == ALIGN
    assert _lf(L, d, ws=P + 64) == ALIGN
    for k in ("q", "k", "v"):
        assert _lf(L, d, o=LFWD[k]) == SHAPE
    for k in ("q", "k", "v", "dout", "dq", "dk", "dv", "log_decay"):
        assert _lb(L, d, **{k: None}) == NULL
        assert _lb(L, d, **{k: LBWD[k] + 1}) == ALIGN
    for k in ("lengths", "s0", "dsT", "ds0"):
        assert _lb(L, d, **{k: P + 2}) == ALIGN
    assert _lb(L, d, ws=P + 64) == ALIGN
    for o in ("dq", "dk", "dv"):
        for k in ("q", "k", "v", "dout", "dq", "dk", "dv"):
            if k != o:
                assert _lb(L, d, **{o: LBWD[k]}) == SHAPE, (o, k)
    assert _lb(L, d, ds0=P + 128, dsT=P + 128) == SHAPE and _lb(L, d, ds0=P + 128, s0=P + 128) == SHAPE
    assert _lf(L, _lin(batch=0), q=None, o=None, log_decay=None) == 0
    assert _lb(L, _lin(batch=0), q=None, dq=None, log_decay=None, ws=None) == 0


def test_linattn_shared_gradients_too_large(L):
    """The gradients of shared keys and values are added up by a thread for four elements: 2^32 at most in a launch."""
    row = Q.HeadStride(0, 1 << 10, 256)
    for length, st in ((1 << 26, LARGE), ((1 << 26) - 256, NULL)):
        d = _lin(batch=1, length=length, heads=2, kv_heads=1, key_width=256,
                 **{n: row for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")})
        assert _lb(L, d, log_decay=None) == st


# ---- norms -------------------------------------------------------------------------------------

def _norm(**kw):
    st = Q.RowStride(3 * 32, 32)
    return Q.NormDesc(**{**dict(dtype=1, rows=5, heads=3, width=32, post=1, pre=1, x=st, gate=st, res=st, h=st, y=st, dy=st,
                                dh=st, dx=st, dgate=st, dres=st, eps=1e-5, alpha=1.0), **kw})


NFWD = dict(x=P, w_post=P + 64, gate=P + S, res=P + 2 * S, w_pre=P + 64, h=P + 3 * S, y=P + 4 * S)
NBWD = dict(x=P, w_post=P + 64, gate=P + S, res=P + 2 * S, w_pre=P + 64, dy=P + 3 * S, dh=P + 4 * S, dx=P + 5 * S,
            dgate=P + 6 * S, dres=P + 7 * S, dw_post=P + 8 * S, dw_pre=P + 9 * S, accumulate=0, ws=P)


def _nf(L, d, **kw):
    return L.pnn_norm_fwd(d, *{**NFWD, **kw}.values(), None)


def _nb(L, d, **kw):
    return L.pnn_norm_bwd(d, *{**NBWD, **kw}.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=-1), DTYPE), (dict(rows=-1), SHAPE), (dict(heads=0), SHAPE), (dict(width=0), SHAPE),
    (dict(width=Q.NORM_MAX_WIDTH + 1), LARGE), (dict(rows=(1 << 30) + 1), LARGE), (dict(heads=1 << 31), LARGE),
    (dict(rows=1 << 20, heads=1 << 11), LARGE), (dict(eps=0.0), VALUE), (dict(eps=-1e-5), VALUE), (dict(eps=NAN), VALUE),
    (dict(eps=INF), VALUE), (dict(eps=1e-40), VALUE), (dict(alpha=NAN), VALUE), (dict(alpha=INF), VALUE)])
def test_norm_descriptions(L, kw, st):
    d = _norm(**kw)
    size = ctypes.c_size_t()
    assert L.pnn_norm_workspace_size(d, ctypes.byref(size)) == st
    assert _nf(L, d) == st and _nb(L, d) == st


def test_norm_arguments(L):
    d = _norm()
    size = ctypes.c_size_t()
    assert L.pnn_norm_workspace_size(None, ctypes.byref(size)) == NULL and L.pnn_norm_workspace_size(d, None) == NULL
    assert L.pnn_norm_workspace_size(d, ctypes.byref(size)) == 0 and size.value > 0
    assert _nf(L, None) == NULL and _nb(L, None) == NULL
    assert _nf(L, d, x=None) == NULL and _nf(L, d, y=None) == NULL and _nf(L, _norm(pre=0), h=None) == NULL
    for k in ("x", "gate", "res", "h", "y"):
        assert _nf(L, d, **{k: NFWD[k] + 1}) == ALIGN
        for s, st in ((Q.RowStride(-96, 32), SHAPE), (Q.RowStride(96, -32), SHAPE), (Q.RowStride(1 << 60, 32), LARGE)):
            assert _nf(L, _norm(**{k: s})) == st
    for k in ("w_post", "w_pre"):
        assert _nf(L, d, **{k: P + 2}) == ALIGN and _nb(L, d, **{k: P + 2}) == ALIGN
    for k in ("h", "y"):
        for s in (Q.RowStride(31, 1000), Q.RowStride(1000, 31), Q.RowStride(90, 32), Q.RowStride(32, 100), Q.RowStride(0, 0)):
            assert _nf(L, _norm(**{k: s})) == SHAPE
    for a, b in (("h", "x"), ("h", "gate"), ("h", "y"), ("y", "x"), ("y", "gate"), ("y", "res")):
        assert _nf(L, d, **{a: NFWD[b]}) == SHAPE
    assert _nf(L, _norm(h=Q.RowStride(96, 40)), h=NFWD["res"]) == SHAPE          # in place, other strides
    assert _nb(L, d, x=None) == NULL and _nb(L, d, dy=None) == NULL and _nb(L, d, ws=None) == NULL
    for k in ("x", "gate", "res", "dy", "dh", "dx", "dgate", "dres"):
        assert _nb(L, d, **{k: NBWD[k] + 1}) == ALIGN
        assert _nb(L, _norm(**{k: Q.RowStride(-96, 32)})) == SHAPE
    for k in ("dw_post", "dw_pre"):
        assert _nb(L, d, **{k: P + 2}) == ALIGN
    assert _nb(L, d, ws=P + 4) == ALIGN
    for k in ("dx", "dgate", "dres"):
        assert _nb(L, _norm(**{k: Q.RowStride(90, 32)})) == SHAPE
        for o in ("x", "gate", "res", "dy", "dh", "dx", "dgate", "dres"):
            if o != k and (k, o) != ("dres", "dh"):
                assert _nb(L, d, **{k: NBWD[o]}) == SHAPE, (k, o)
    assert _nb(L, _norm(dres=Q.RowStride(96, 40)), dres=NBWD["dh"]) == SHAPE
    assert _nb(L, d, dw_post=NBWD["dw_pre"]) == SHAPE
    assert _nf(L, _norm(rows=0), x=None, h=None, y=None) == 0
    # nothing wanted: nothing done
    assert _nb(L, d, x=None, dx=None, dgate=None, dres=None, dw_post=None, dw_pre=None) == 0


def test_norm_weight_gradients_in_place_of_weights(L):
    for k in ("dw_post", "dw_pre"):
        for w in ("w_post", "w_pre"):
            assert _nb(L, _norm(), **{k: NBWD[w]}) == SHAPE, (k, w)


# ---- policy loss -------------------------------------------------------------------------------

def _policy(**kw):
    return Q.PolicyDesc(**{**dict(dtype=1, rows=4, classes=32, logit_stride=32, grad_stride=32, temperature=0.7,
                                  clip_low=0.2, clip_high=0.3, kl=0.1, scale=0.25), **kw})


POL = dict(z=P, tokens=P + S, advantage=P + 2 * S, old=P + 3 * S, ref=P + 4 * S, weight=P + 5 * S, loss=P + 6 * S,
           logp=P + 7 * S, dz=P + 8 * S)


def _pol(L, d, **kw):
    return L.pnn_policy_fwd_bwd(d, *{**POL, **kw}.values(), None)


@pytest.mark.parametrize("kw,st", [
    (dict(dtype=3), DTYPE), (dict(rows=-1), SHAPE), (dict(classes=0), SHAPE), (dict(logit_stride=-1), SHAPE),
    (dict(grad_stride=31), SHAPE), (dict(rows=(1 << 28) + 1), LARGE), (dict(classes=1 << 31), LARGE),
    (dict(logit_stride=1 << 60), LARGE), (dict(temperature=0.0), VALUE), (dict(temperature=-1.0), VALUE),
    (dict(temperature=NAN), VALUE), (dict(temperature=INF), VALUE), (dict(temperature=1e-40), VALUE),
    (dict(clip_low=-0.1), VALUE), (dict(clip_high=-0.1), VALUE), (dict(clip_low=NAN), VALUE), (dict(clip_high=INF), VALUE),
    (dict(kl=NAN), VALUE), (dict(scale=INF), VALUE), (dict(scale=1e30, temperature=1e-30), VALUE)])
def test_policy_descriptions(L, kw, st):
    assert _pol(L, _policy(**kw)) == st


def test_policy_arguments(L):
    d = _policy()
    assert _pol(L, None) == NULL
    for k in ("z", "tokens", "advantage", "ref", "loss"):
        assert _pol(L, d, **{k: None}) == NULL
    for k in POL:
        assert _pol(L, d, **{k: POL[k] + 1}) == ALIGN
    assert _pol(L, _policy(grad_stride=40), dz=POL["z"]) == SHAPE
    assert _pol(L, d, logp=POL["loss"]) == SHAPE
    assert _pol(L, _policy(rows=0), z=None, loss=None) == 0


def test_policy_outputs_in_place_of_inputs(L):
    for k in ("loss", "logp"):
        for o in ("advantage", "old", "ref", "weight"):
            assert _pol(L, _policy(), **{k: POL[o]}) == SHAPE, (k, o)


def test_python_descriptions():
    import torch
    q, v = torch.zeros(2, 5, 4, 8), torch.zeros(2, 5, 2, 6)
    k, o = torch.zeros(2, 5, 2, 8), torch.zeros(2, 5, 4, 6)
    d = Q.linattn_desc(q, k, v, o, scale=0.5)
    assert (d.heads, d.kv_heads, d.key_width, d.value_width, d.o.step, d.dq.step) == (4, 2, 8, 6, 24, 0)
    for bad in ((q, k, v, q), (q, k[:, :4], v, o), (q, k.bfloat16(), v, o), (q[0], k, v, o),
                (q.transpose(2, 3), k, v, o), (q, k, v, o, o.bfloat16())):
        with pytest.raises(ValueError):
            Q.linattn_desc(*bad)
    with pytest.raises(TypeError):
        Q.linattn_desc(q.half(), k.half(), v.half(), o.half())
    x = torch.zeros(5, 8)
    d = Q.norm_desc(x, y=x, pre=True)
    assert (d.rows, d.heads, d.width, d.x.row, d.post, d.pre, d.h.row) == (5, 1, 8, 8, 0, 1, 0)
    d = Q.norm_desc(torch.zeros(5, 4, 8).transpose(0, 1), post=1)
    assert (d.rows, d.heads, d.x.row, d.x.head) == (4, 5, 8, 32)
    for bad in (dict(h=x[:4]), dict(gate=x.bfloat16()), dict(y=x.t())):
        with pytest.raises(ValueError):
            Q.norm_desc(x, **bad)
    with pytest.raises(ValueError):
        Q.norm_desc(x[0])
    with pytest.raises(ValueError):
        Q.policy_desc(x, x[:4])
    with pytest.raises(ValueError):
        Q.policy_desc(x, x.bfloat16())
    assert Q.policy_desc(x).grad_stride == 8
