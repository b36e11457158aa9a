"""The norms' backward from the sum that the forward stored: after a forward in place, where nothing else is left, and
beside the residual, against 64 bits; with the residual kept, the gradients that it gives."""
from unittest import mock

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import f64
from tests.test_gpu_norm import EPS, Case, _checked, _seq, _stream

pytestmark = pytest.mark.gpu


def _describe(c, **kw):
    t = dict(gate=c.gate, res=c.res, h=c.h, y=c.y, dy=c.dy, dh=c.dh, dx=c.dx, dgate=c.dgate, dres=c.dres, post=c.post,
             pre=c.pre, eps=EPS, alpha=c.alpha)
    return _seq().norm_desc(c.x, **{**t, **kw})


def _backward(c, desc, given, x="x"):
    s = _seq()
    ws = torch.full((max(s.pnn_norm_workspace_size(desc), 256),), 0xCD, dtype=torch.uint8, device="cuda")
    one = lambda f: None if f is None else f.t[0]
    s.pnn_norm_bwd(desc, getattr(c, x) if x else None, c.w1, c.gate, given, c.w2, c.dy, c.dh, c.dx, c.dgate, c.dres,
                   one(c.f1), one(c.f2), False, ws, _stream())


def _at_the_stored_sum(c, h):
    """block_ref's backward with h as it is stored, exactly."""
    h = f64(h)
    with mock.patch.object(R, "norm_fwd", lambda *a: {"h": (h, torch.zeros_like(h))}):
        return c.reference()


CASES = [
    # rows, heads, width, dtype, parts, lead, pad, swap
    (1, 1, 1, "f32", "pgrnwd", 0, 0, False),
    (5, 1, 7, "bf16", "pgrnwd", 1, 2, False),
    (40, 2, 129, "bf16", "pgrnwd", 5, 0, False),
    (33, 3, 64, "f32", "prnw", 3, 1, True),
    (9, 1, 515, "f32", "pgrnwd", 0, 0, False),
    (19, 1, 257, "bf16", "rnwd", 0, 0, False),
    (30, 1, 1000, "bf16", "grnw", 0, 0, False),
    (700, 1, 2048, "bf16", "prnwd", 0, 0, False),
    (1100, 1, 2056, "bf16", "pgrnwd", 0, 0, False),
    (3, 1, 2050, "f32", "prnwd", 0, 0, False),
    (2, 1, 8191, "bf16", "pgrnwd", 2, 1, False),
    (2, 1, 16383, "f32", "pgrnwd", 0, 0, False),
]


@pytest.mark.parametrize("rows,heads,width,dtype,parts,lead,pad,swap", CASES)
def test_after_a_forward_in_place(rows, heads, width, dtype, parts, lead, pad, swap):
    c = Case(rows, heads, width, dtype, parts, lead, pad, swap)
    whole = c.reference()                        # while the residual is there
    desc = _describe(c, h=c.res, stored=True)
    _seq().pnn_norm_fwd(desc, c.x, c.w1, c.gate, c.res, c.w2, c.res, c.y, _stream())
    _backward(c, desc, c.res)
    c.check_backward(_at_the_stored_sum(c, c.res))
    if dtype == "f32":                           # the sum's rounding is within the bounds of forming it again
        c.check_backward(whole)
    c.intact()


@pytest.mark.parametrize("rows,heads,width,dtype,parts,lead,pad,swap", CASES)
def test_sum_beside_the_residual(rows, heads, width, dtype, parts, lead, pad, swap):
    c = Case(rows, heads, width, dtype, parts, lead, pad, swap)
    c.forward()
    c.res.fill_(7.0)                             # not looked at
    ref = _at_the_stored_sum(c, c.h)
    desc = _describe(c, stored=True)
    _backward(c, desc, c.h)
    c.check_backward(ref)
    if not c.post and c.gate is None:            # nor is x
        for n in ("dx", "dres"):
            getattr(c, n).fill_(3.0)
        _backward(c, desc, c.h, x=None)
        c.check_backward(ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sum_without_a_residual(dtype):
    c = Case(37, 2, 72, dtype, "pnwd")
    c.forward()
    _backward(c, _describe(c, stored=True), c.h)
    c.check_backward(_at_the_stored_sum(c, c.h))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("parts", ["pgrnwd", "pnwd"])
def test_kept_parts_of_the_sum(dtype, parts):
    """Given h, a description with kept has the gradients that the residual gives, bit by bit."""
    c = Case(50, 1, 520, dtype, parts)
    c.forward()
    c.backward()
    names = [n for n in ("dx", "dgate", "dres") if getattr(c, n) is not None]
    want = [getattr(c, n).clone() for n in names] + [c.f1.t.clone(), c.f2.t.clone()]
    for t in [getattr(c, n) for n in names] + [c.f1.t, c.f2.t]:
        t.fill_(5.0)
    _backward(c, _describe(c, kept=True), c.h)
    for t, w in zip([getattr(c, n) for n in names] + [c.f1.t, c.f2.t], want):
        assert torch.equal(t, w)
    ref = c.reference()
    for n in names:
        _checked(n, getattr(c, n), ref[n], dtype)


def test_in_place_in_a_graph():
    c = Case(700, 1, 520, "bf16", "pgrnwd")
    s = _seq()
    desc = _describe(c, h=c.res, stored=True)
    ws = torch.empty(s.pnn_norm_workspace_size(desc), dtype=torch.uint8, device="cuda")
    first, outs = c.res.clone(), [c.res, c.y, c.dx, c.dgate, c.dres, c.f1.t, c.f2.t]

    def both():
        s.pnn_norm_fwd(desc, c.x, c.w1, c.gate, c.res, c.w2, c.res, c.y, _stream())
        s.pnn_norm_bwd(desc, c.x, c.w1, c.gate, c.res, c.w2, c.dy, c.dh, c.dx, c.dgate, c.dres, c.f1.t[0], c.f2.t[0],
                       False, ws, _stream())

    both()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in outs[1:]:
            t.fill_(5.0)
        ws.fill_(0x77)
        c.res.copy_(first)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outs, want))
