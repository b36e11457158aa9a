"""Norms around a block where their inputs are at their ends: rows of zeros, infinite gates, values that are not finite,
parts left out, results in place, offsets past 2^31, streams and graphs; gradients against difference quotients."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import within
from tests.test_gpu_norm import EPS, Case, _seq, _stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [24, 700, 3000, 9000])
def test_rows_of_zeros_and_tiny_and_large_values(dtype, width):
    c = Case(6, 1, width, dtype, "pgrnwd")
    for t in (c.x, c.res):
        t[0] = 0.0
        t[1] *= 1e-18
        t[2] *= 1e15
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward(c.reference())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_at_their_ends(dtype):
    """silu(-inf) = 0 with slope 0; +inf: an infinite output where a is not 0, slope 1."""
    c = Case(4, 1, 40, dtype, "pgw")
    c.gate[0, 0, :8] = -math.inf
    c.gate[1, 0, :8] = -200.0
    c.gate[2, 0, :8] = 100.0
    c.forward()
    c.check_forward()
    c.desc.dh = c.desc.x                                # dh: h's gradient, here the x
    c.dh = c.x
    c.backward()
    c.check_backward(R.norm_bwd(c.x, c.w_post, c.gate, None, None, None, c.x, True, False, c.desc.eps, c.alpha))
    assert not c.h[0, 0, :8].any() and not c.dgate[0, 0, :8].any()
    c.gate[3, 0, 0] = math.inf
    c.forward()
    assert torch.isinf(c.h[3, 0, 0]) and torch.isfinite(c.h[3, 0, 1:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_in_their_row(dtype):
    for heads, width in ((4, 32), (1, 600), (1, 5000)):
        clean, dirty = (Case(9, heads, width, dtype, "pgrnwd", seed=3) for _ in range(2))
        dirty.x[2, 0, 5] = math.nan
        dirty.res[4, 0, 7] = math.inf
        for c in (clean, dirty):
            c.forward()
            c.backward()
        rows = [r for r in range(9) if r not in (2, 4)]
        for n in ("h", "y", "dx", "dgate", "dres"):
            assert torch.equal(getattr(clean, n)[rows], getattr(dirty, n)[rows]), n
            if heads > 1:
                assert torch.equal(getattr(clean, n)[:, 1:], getattr(dirty, n)[:, 1:]), n
        assert torch.isnan(dirty.y[2, 0]).all()


def test_no_rows():
    c = Case(0, 1, 40, "bf16", "prnwd")
    c.forward()
    before = [f.t[0].clone() for f in (c.f1, c.f2)]
    c.backward(accumulate=True)
    assert all(torch.equal(f.t[0], b) for f, b in zip((c.f1, c.f2), before))
    c.backward()
    assert not c.f1.t.any() and not c.f2.t.any()


def test_parts_left_out():
    """Gradients one at a time have the bits they have together; results that are not wanted stay as they were."""
    c = Case(50, 2, 96, "bf16", "pgrnwd")
    s = _seq()
    c.forward()
    y = c.y.clone()
    c.y.zero_()
    s.pnn_norm_fwd(c.desc, c.x, c.w1, c.gate, c.res, c.w2, None, c.y, _stream())
    assert torch.equal(c.y, y)
    c.backward()
    names = ("dx", "dgate", "dres", "dw_post", "dw_pre")
    get = lambda n: {"dw_post": c.f1.t[0], "dw_pre": c.f2.t[0]}[n] if n.startswith("dw") else getattr(c, n)
    want = {n: get(n).clone() for n in names}
    ws = torch.empty(s.pnn_norm_workspace_size(c.desc), dtype=torch.uint8, device="cuda")
    for only in names:
        for n in names:
            get(n).fill_(3.0)
        a = {n: get(n) if n == only else None for n in names}
        s.pnn_norm_bwd(c.desc, c.x, c.w1, c.gate, c.res, c.w2, c.dy, c.dh, a["dx"], a["dgate"], a["dres"], a["dw_post"],
                       a["dw_pre"], False, ws if only.startswith("dw") else None, _stream())
        for n in names:
            assert torch.equal(get(n), want[n]) if n == only else bool((get(n) == 3.0).all()), (only, n)


@pytest.mark.parametrize("dtype,width,parts", [("bf16", 2048, "prnw"), ("f32", 129, "rn"), ("bf16", 72, "pgr")])
def test_the_sum_in_the_residuals_place(dtype, width, parts):
    c = Case(300, 1, width, dtype, parts, pad=3)
    c.forward()
    h, y = c.h.clone(), None if c.y is None else c.y.clone()
    s = _seq()
    s.pnn_norm_fwd(c.desc, c.x, c.w1, c.gate, c.res, c.w2, c.res, c.y, _stream())
    assert torch.equal(c.res, h) and (y is None or torch.equal(c.y, y))
    c.intact()


def test_gradient_without_a_norm_or_gate():
    """dx = alpha dh, dres = dh; x is not looked at."""
    c = Case(20, 1, 33, "f32", "rd")
    _seq().pnn_norm_bwd(c.desc, None, None, None, None, None, None, c.dh, c.dx, None, c.dres, None, None, False, None,
                        _stream())
    assert torch.equal(c.dx, c.alpha * c.dh) and torch.equal(c.dres, c.dh)


def test_without_a_gradient_of_the_sum():
    c = Case(20, 1, 256, "bf16", "pgrnw")
    c.forward()
    c.backward()
    c.check_backward(c.reference())
    c = Case(20, 1, 256, "bf16", "pg")                  # no gradient reaches it at all
    c.backward()
    assert not c.dx.any() and not c.dgate.any() and not c.f1.t.any()


def test_offsets_past_2_31_elements():
    rows, gap = 40, 1 << 26
    buf = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda")
    c = Case(rows, 1, 48, "bf16", "pgrnwd")
    far = [buf.as_strided((rows, 1, 48), (gap, 48, 1), 64 * i) for i in range(4)]
    far[0].copy_(c.x)
    far[1].copy_(c.dy)
    s = _seq()
    c.x, c.dy, c.y, c.dx = far[0], far[1], far[2], far[3]
    c.desc = s.norm_desc(c.x, gate=c.gate, res=c.res, h=c.h, y=c.y, dy=c.dy, dh=c.dh, dx=c.dx, dgate=c.dgate, dres=c.dres,
                         post=True, pre=True, eps=EPS, alpha=c.alpha)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward(c.reference())


def test_other_streams_and_graph_replays():
    c = Case(700, 1, 520, "bf16", "pgrnwd")
    s = _seq()
    ws = torch.empty(s.pnn_norm_workspace_size(c.desc), dtype=torch.uint8, device="cuda")
    names = ("h", "y", "dx", "dgate", "dres")

    def both():
        c.forward()
        s.pnn_norm_bwd(c.desc, c.x, c.w1, c.gate, c.res, c.w2, c.dy, c.dh, c.dx, c.dgate, c.dres, c.f1.t[0], c.f2.t[0],
                       False, ws, _stream())

    both()
    want = [getattr(c, n).clone() for n in names] + [c.f1.t.clone(), c.f2.t.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in [getattr(c, n) for n in names] + [c.f1.t, c.f2.t]:
            t.fill_(5.0)
        ws.fill_(0x77)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip([getattr(c, n) for n in names] + [c.f1.t, c.f2.t], want):
            assert torch.equal(t, w)


def test_gradients_against_difference_quotients():
    """fp32: central differences of step e leave (e^2 / 6) times the third derivative, some 1e-6 of the slope at
    e = 2^-9 for these sizes, and the forward's rounding, 2^-22 of the loss's magnitude, over e: 2^-13 of the summed
    magnitudes."""
    c = Case(3, 1, 20, "f32", "pgrnwd")
    c.forward()
    c.backward()
    e = 2.0 ** -9
    g = torch.Generator().manual_seed(1)
    loss = lambda: float((R.f64(c.h) * R.f64(c.dh)).sum() + (R.f64(c.y) * R.f64(c.dy)).sum())
    size = float((R.f64(c.h) * R.f64(c.dh)).abs().sum() + (R.f64(c.y) * R.f64(c.dy)).abs().sum())
    for t, grad in ((c.x, c.dx), (c.gate, c.dgate), (c.res, c.dres), (c.w1, c.f1.t[0]), (c.w2, c.f2.t[0])):
        way = torch.randn(t.shape, generator=g).cuda()
        got = float((R.f64(grad) * R.f64(way)).sum())
        keep, ends = t.clone(), []
        for sign in (1, -1):
            t.copy_(keep + sign * e * way)
            c.forward()
            ends.append(loss())
        t.copy_(keep)
        assert abs((ends[0] - ends[1]) / (2 * e) - got) <= 2.0 ** -13 * size + 1e-4 * abs(got) + 1e-4 * size
