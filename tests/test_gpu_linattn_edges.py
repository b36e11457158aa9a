"""Linear attention where its inputs are at their ends: decays of 0 and -inf, values that are not finite, empty and single
steps, states in place, offsets past 2^31, other streams, graphs; gradients against difference quotients."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import DT, within
from tests.test_gpu_linattn import Case, _seq, _stream, _ws

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 5, 33, 300])
def test_decays_at_their_ends(dtype, T):
    """0: a plain sum; -inf and -1e30: nothing is kept; -1e-9: hardly anything is lost.  Heads with a positive or NaN decay
    are NaN, the others stay."""
    c = Case(2, T, 6, 3, 24, 40, dtype)
    c.decay.copy_(torch.tensor([0.0, -math.inf, -1e30, -1e-9, -5.0, -0.1]))
    c.forward()
    c.backward()
    c.check(c.reference())
    names = [n for n in ("o", "sT", "dq", "ds0")]
    first = [getattr(c, n).clone() for n in names]
    c.decay[0], c.decay[5] = 0.5, math.nan
    c.forward()
    c.backward()
    for n, t in zip(names, first):
        heads = 1 if n in ("sT", "ds0") else 2
        got = getattr(c, n)
        assert torch.isnan(got.select(heads, 0)).all() and torch.isnan(got.select(heads, 5)).all(), n
        assert torch.equal(got.narrow(heads, 1, 4), t.narrow(heads, 1, 4)), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(dtype, what, value):
    """Reach their own step and later ones, in their sequence and head; backwards in time earlier ones.  Others keep their
    bits."""
    clean, dirty = (Case(2, 150, 2, 2, 40, 64, dtype, seed=2) for _ in range(2))
    at, b, h = 77, 1, 1
    getattr(dirty, what)[b, at, h, 3] = value
    for c in (clean, dirty):
        c.forward()
        c.backward()
    same = lambda n, *ix: torch.equal(getattr(clean, n)[ix], getattr(dirty, n)[ix])
    for n in ("o", "sT", "dq", "dk", "dv", "ds0"):
        assert same(n, 1 - b) and (same(n, slice(None), slice(None), 1 - h) if n not in ("sT", "ds0")
                                   else same(n, slice(None), 1 - h)), n
    early, late = slice(0, at), slice(at + 1, None)
    lost = lambda t: not torch.isfinite(t).any()
    assert same("o", b, early, h)
    if what == "q":
        assert lost(dirty.o[b, at, h]) and same("o", b, late, h) and same("sT") and same("dq")
        assert same("dk", b, late, h) and same("dv", b, late, h)
        assert lost(dirty.dv[b, :at + 1, h]) and lost(dirty.dk[b, :at + 1, h, 3])
    if what == "k":
        assert lost(dirty.o[b, at:, h]) and lost(dirty.sT[b, h, 3])
        assert same("dq", b, early, h) and lost(dirty.dq[b, at:, h, 3])
        assert same("dk") and same("dv", b, late, h) and same("dv", b, early, h) and lost(dirty.dv[b, at, h])
    if what == "v":
        assert lost(dirty.o[b, at:, h, 3]) and lost(dirty.sT[b, h, :, 3])
        assert same("dq", b, early, h) and lost(dirty.dq[b, at:, h])
        assert same("dv") and same("dk", b, late, h) and same("dk", b, early, h) and lost(dirty.dk[b, at, h])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_behind_a_sequence_are_not_looked_at(dtype):
    clean, dirty = (Case(3, 130, 2, 1, 33, 70, dtype, ragged=True, seed=9) for _ in range(2))
    for b, n in enumerate(clean.lengths.tolist()):
        n = max(0, min(n, 130))
        for t in ("q", "k", "v", "dout"):
            getattr(dirty, t)[b, n:] = math.nan
    for c in (clean, dirty):
        c.forward()
        c.backward()
    for n in ("o", "sT", "dq", "dk", "dv", "ds0"):
        assert torch.equal(getattr(clean, n), getattr(dirty, n)), n
    for b, n in enumerate(clean.lengths.tolist()):
        n = max(0, min(n, 130))
        for t in ("o", "dq", "dk", "dv"):
            assert not getattr(dirty, t)[b, n:].any()
        if n == 0:
            assert torch.equal(dirty.sT[b], dirty.s0[b]) and torch.equal(dirty.ds0[b], dirty.dsT[b])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_lowest_values(dtype):
    """Values of 1e15 and 2^-60: no factor on the way leaves the range.  Three factors of 1e15 do: then the result is not
    finite."""
    for size in (1e15, 2.0 ** -60):
        c = Case(1, 70, 2, 2, 16, 24, dtype, state=False)
        for t in (c.q, c.k, c.v, c.dout):
            t.mul_(size if t is not c.q else 1.0)
        c.forward()
        c.backward()
        ref = c.reference()
        if size > 1:                                  # dq: do, v and k, 1e45
            assert ref.pop("dq")[0].abs().median() > 1e40 and not torch.isfinite(c.dq).any()
        c.check(ref)


def test_no_steps():
    for state in (True, False):
        c = Case(2, 0, 2, 1, 16, 24, "bf16", state=state)
        c.forward()
        c.backward()
        if state:
            assert torch.equal(c.sT, c.s0) and torch.equal(c.ds0, c.dsT)
    c = Case(2, 0, 2, 1, 16, 24, "bf16")
    s = _seq()
    s.pnn_linattn_fwd(c.desc, None, None, None, c.decay, None, None, None, c.sT, None, _stream())
    assert not c.sT.any()


@pytest.mark.parametrize("dtype,B,T,H,kv,K,V", [
    ("bf16", 64, 1, 16, 16, 128, 128), ("f32", 3, 1, 4, 2, 65, 33), ("bf16", 2, 1, 5, 1, 256, 250), ("f32", 300, 1, 8, 8, 7, 3),
    ("bf16", 2, 400, 3, 3, 64, 128), ("f32", 40, 65, 16, 4, 16, 130), ("bf16", 80, 64, 8, 8, 128, 256)])
def test_states_in_place(dtype, B, T, H, kv, K, V):
    """sT = s0, with more workgroups than run at a time; the same bits as apart."""
    c = Case(B, T, H, kv, K, V, dtype, ragged=B > 2)
    c.forward()
    o, sT = c.o.clone(), c.sT.clone()
    c.o.fill_(9.0)
    c.forward(s0="s0", sT="s0")
    assert torch.equal(c.o, o) and torch.equal(c.s0, sT)
    if B * T * H * K * V < 1 << 25:
        c.fs["s0"].t.copy_(torch.randn(c.s0.shape, generator=c.g))
        c.forward()
        ref = c.reference(backward=False)
        c.check(ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_step_at_a_time_is_the_whole_sequence(dtype):
    """The single-step form over 40 steps against the definition; and its state against the chunked form's."""
    c = Case(3, 40, 4, 2, 48, 36, dtype, ragged=True)
    ref = c.reference(backward=False)
    s = _seq()
    state = c.s0.clone()
    out = torch.empty_like(c.o)
    for t in range(40):
        q, k, v, o = (x[:, t:t + 1] for x in (c.q, c.k, c.v, out))
        live = (c.lengths > t).to(torch.int32)
        d = s.linattn_desc(q, k, v, o, scale=c.scale)
        s.pnn_linattn_fwd(d, q, k, v, c.decay, live, state, o, state, None, _stream())
    within(out, *ref["o"], dtype)
    within(state, *ref["sT"], "f32")


def test_first_state_without_a_last_and_the_other_way_round():
    c = Case(2, 90, 2, 2, 32, 32, "bf16")
    s = _seq()
    for T in (90, 1):
        d = s.linattn_desc(c.q[:, :T], c.k[:, :T], c.v[:, :T], c.o[:, :T], scale=c.scale)
        ws = _ws(s.pnn_linattn_sizes(d)[0])
        for s0, sT in ((c.s0, None), (None, c.sT), (None, None)):
            s.pnn_linattn_fwd(d, c.q, c.k, c.v, c.decay, None, s0, c.o, sT, ws, _stream())
            ref = R.linattn(c.q[:, :T], c.k[:, :T], c.v[:, :T], c.decay, None, s0, d.scale, "bf16")
            within(c.o[:, :T], *ref["o"], "bf16")
            if sT is not None:
                within(sT, *ref["sT"], "f32")
    for s0, dsT, ds0 in ((c.s0, None, None), (None, c.dsT, None), (None, None, c.ds0)):
        s.pnn_linattn_bwd(c.desc, c.q, c.k, c.v, c.decay, None, s0, c.dout, dsT, c.dq, c.dk, c.dv, ds0,
                          _ws(s.pnn_linattn_sizes(c.desc)[1]), _stream())
        ref = R.linattn(c.q, c.k, c.v, c.decay, None, s0, c.desc.scale, "bf16", c.dout, dsT)
        for n in ("dq", "dk", "dv"):
            within(getattr(c, n), *ref[n], "bf16")
        if ds0 is not None:
            within(ds0, *ref["ds0"], "f32")


def test_broadcast_inputs():
    """A stride of zero reads the same values for every head, step or sequence; gradients stay apart."""
    c = Case(2, 50, 4, 4, 16, 16, "f32")
    s = _seq()
    q = c.q[:, :, :1].expand(2, 50, 4, 16)
    k = c.k[:1, :1].expand(2, 50, 4, 16)
    d = s.linattn_desc(q, k, c.v, c.o, c.dout, c.dq, c.dk, c.dv, scale=c.scale)
    s.pnn_linattn_fwd(d, q, k, c.v, c.decay, None, c.s0, c.o, c.sT, _ws(s.pnn_linattn_sizes(d)[0]), _stream())
    s.pnn_linattn_bwd(d, q, k, c.v, c.decay, None, c.s0, c.dout, c.dsT, c.dq, c.dk, c.dv, c.ds0,
                      _ws(s.pnn_linattn_sizes(d)[1]), _stream())
    c.check(R.linattn(q, k, c.v, c.decay, None, c.s0, d.scale, "f32", c.dout, c.dsT))


def test_offsets_past_2_31_elements():
    """Steps 2^26 elements apart: step 32 starts at 2^31."""
    T, gap = 40, 1 << 26
    buf = torch.empty(T * gap, dtype=torch.bfloat16, device="cuda")
    c = Case(1, T, 1, 1, 16, 24, "bf16")
    s = _seq()
    far = lambda w, at: buf.as_strided((1, T, 1, w), (0, gap, 0, 1), at)
    q, k, v, o, dq = far(16, 0), far(16, 64), far(24, 128), far(24, 192), far(16, 256)
    for x, y in ((q, c.q), (k, c.k), (v, c.v)):
        x.copy_(y)
    d = s.linattn_desc(q, k, v, o, c.dout, dq, c.dk, c.dv, scale=c.scale)
    s.pnn_linattn_fwd(d, q, k, v, c.decay, None, c.s0, o, c.sT, _ws(s.pnn_linattn_sizes(d)[0]), _stream())
    s.pnn_linattn_bwd(d, q, k, v, c.decay, None, c.s0, c.dout, c.dsT, dq, c.dk, c.dv, c.ds0,
                      _ws(s.pnn_linattn_sizes(d)[1]), _stream())
    c.o, c.dq = o, dq
    c.check(c.reference())


def test_other_streams_side_by_side():
    cases = [Case(2, 300, 2, 1, 64, 96, "bf16", seed=i) for i in range(2)]
    want = []
    for c in cases:
        c.forward()
        c.backward()
        want.append([getattr(c, n).clone() for n in ("o", "sT", "dq", "dk", "dv", "ds0")])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c, st in zip(cases, streams):
            with torch.cuda.stream(st):
                c.forward()
                c.backward()
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        for n, t in zip(("o", "sT", "dq", "dk", "dv", "ds0"), w):
            assert torch.equal(getattr(c, n), t)


def test_graph_replays():
    c = Case(3, 200, 4, 2, 64, 80, "bf16", ragged=True)
    s = _seq()
    ws = _ws(max(s.pnn_linattn_sizes(c.desc)))

    def both():
        s.pnn_linattn_fwd(c.desc, c.q, c.k, c.v, c.decay, c.lengths, c.s0, c.o, c.sT, ws, _stream())
        s.pnn_linattn_bwd(c.desc, c.q, c.k, c.v, c.decay, c.lengths, c.s0, c.dout, c.dsT, c.dq, c.dk, c.dv, c.ds0, ws,
                          _stream())

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    names = ("o", "sT", "dq", "dk", "dv", "ds0")
    for i in range(3):
        c.q.mul_(0.9)                              # other inputs and lengths, the same addresses
        c.lengths.copy_(torch.tensor([200, 50 * i, 199 - i], dtype=torch.int32))
        both()
        want = [getattr(c, n).clone() for n in names]
        for n in names:
            getattr(c, n).fill_(5.0)
        ws.fill_(0x77)
        graph.replay()
        torch.cuda.synchronize()
        for n, t in zip(names, want):
            assert torch.equal(getattr(c, n), t), n


def test_gradients_against_difference_quotients():
    """fp32.  The loss is linear in each of q, k, v and s0 alone, so a difference quotient has no error of its own: what is
    left are the rounding of two losses (sums of 2 x 45 x 2 x 20 outputs, bound as in block_ref) and of the gradient."""
    c = Case(2, 45, 2, 1, 12, 20, "f32")
    c.forward()
    c.backward()
    g = torch.Generator().manual_seed(5)
    value = lambda r: (float((r["o"][0] * R.f64(c.dout)).sum() + (r["sT"][0] * R.f64(c.dsT)).sum()))
    size = lambda r: (float((r["o"][1] * R.f64(c.dout).abs()).sum() + (r["sT"][1] * R.f64(c.dsT).abs()).sum()))
    ref = c.reference()
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("s0", "ds0")):
        t = getattr(c, name)
        way = torch.randn(t.shape, generator=g).cuda()
        got = float((R.f64(getattr(c, grad)) * R.f64(way)).sum())
        keep = t.clone()
        ends, slack = [], 0.0
        for sign in (1, -1):
            t.copy_(keep + sign * 0.5 * way)
            moved = R.f64(t) - R.f64(keep)                    # as rounded
            c.forward()
            r = {"o": (R.f64(c.o), None), "sT": (R.f64(c.sT), None)}
            ends.append(value(r))
            slack += size(c.reference(backward=False)) + float((R.f64(getattr(c, grad)).abs() *
                                                                (moved - sign * 0.5 * R.f64(way)).abs()).sum())
        t.copy_(keep)
        slack += float((ref[grad][1] * R.f64(way).abs()).sum()) + 1e-6 * abs(got)
        assert abs(ends[0] - ends[1] - got) <= slack, (name, ends[0] - ends[1], got, slack)
