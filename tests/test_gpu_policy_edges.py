"""The policy loss where its inputs are at their ends: clipped rows, logits of -inf and the type's lowest value, values
that are not finite, masked rows, offsets past 2^31, streams and graphs; gradients against difference quotients."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import DT, within
from tests.test_gpu_policy import HIGH, LOW, Case, _seq, _stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 3000, 9001])
def test_clipped_rows(dtype, V):
    """Ratios below, within and above the bounds, advantages of either sign and 0: the gradient of the unclipped term where
    it is the smaller one, none otherwise."""
    c = Case(9, V, dtype, kl=0.0, masked=False)
    lp = torch.log_softmax(c.z.cpu().double(), 1)[torch.arange(9), c.tokens.cpu().long()]
    off = torch.tensor([-1.0, 0.0, 1.0] * 3)
    c.old.copy_((lp - off).float())
    c.advantage.copy_(torch.tensor([1.0] * 3 + [-1.0] * 3 + [0.0] * 3))
    c.run()
    c.check(c.reference())
    for r, clipped in enumerate([0, 0, 1, 1, 0, 0, 1, 1, 1]):
        assert bool(c.dlogits[r].any()) != bool(clipped), r
    want = torch.tensor([-math.exp(-1), -1.0, -(1 + HIGH), 1 - LOW, 1.0, math.e, 0, 0, 0])
    assert torch.allclose(c.loss.cpu(), want, rtol=1e-4, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 5000, 70000 * 2])
def test_logits_at_their_ends(dtype, V):
    """Classes of -inf have no probability and no gradient; of the type's lowest value neither; a row of nothing but -inf
    or with a NaN or an infinity is NaN; rows of equal lowest or huge values are uniform."""
    c = Case(9, V, dtype, kl=0.1, masked=False)
    low = torch.finfo(DT[dtype]).min
    a = c.tokens.clone()
    z = c.z
    z[0, ::2] = -math.inf
    z[0, a[0]] = 1.0
    z[1] = low
    z[1, a[1]] = 0.5
    z[2] = low
    z[3] = -math.inf
    z[4, V // 3] = math.nan
    z[5, V // 2] = math.inf
    z[6] = 3e38
    z[7] = -math.inf
    z[7, a[7]] = 2.0
    z[8, :V // 2] = -math.inf                    # a whole stretch, so that a thread sees nothing else
    z[8, a[8]] = 0.0
    lp = torch.log_softmax(z.cpu().double(), 1)[torch.arange(9), a.cpu().long()]
    c.old.copy_(torch.nan_to_num(lp - 0.05, nan=0.0).float())
    c.ref.copy_(torch.nan_to_num(lp + 0.1, nan=0.0).float())
    ref = c.reference()
    c.run()
    c.check(ref)
    assert torch.isnan(c.loss[3:6]).all() and torch.isnan(c.dlogits[3:6].float()).all()
    assert not c.dlogits[0][z[0] == -math.inf].any() and not c.dlogits[7].any() and c.logp[7] == 0.0


def test_a_token_without_probability():
    """log p = -inf: the ratio is 0, the loss of the KL term infinite, without it 0."""
    c = Case(1, 30, "f32", kl=0.0, masked=False)
    c.z[0, c.tokens[0]] = -math.inf
    c.old.fill_(-1.0)
    c.run()
    assert c.logp[0] == -math.inf and c.loss[0].abs() <= 0.8 * c.advantage[0].abs() and torch.isfinite(c.dlogits).all()


def test_masked_rows_are_not_looked_at():
    for V in (33, 2500, 70001):
        clean, dirty = (Case(12, V, "bf16", seed=1) for _ in range(2))
        mask = clean.tokens < 0
        assert mask.any() and not mask.all()
        for t in (dirty.z, dirty.old, dirty.ref, dirty.advantage, dirty.weight):
            t[mask] = math.nan
        for c in (clean, dirty):
            c.run()
        same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=7.0), torch.nan_to_num(b.float(), nan=7.0))
        for n in ("loss", "logp", "dlogits"):
            assert same(getattr(clean, n), getattr(dirty, n))
            assert not getattr(dirty, n)[mask].any()


def test_all_rows_masked_and_no_rows():
    c = Case(7, 100, "bf16")
    c.tokens.fill_(-1)
    c.run()
    assert not c.loss.any() and not c.logp.any() and not c.dlogits.any()
    s = _seq()
    d = s.policy_desc(c.z[:0], c.dlogits[:0])
    s.pnn_policy_fwd_bwd(d, None, None, None, None, None, None, None, None, None, _stream())


def test_sure_policies():
    """A probability of nearly 1: its token's gradient is that of 1 - p, which is formed from the logarithm."""
    c = Case(4, 200, "f32", kl=0.0, old=False, masked=False, weight=False)
    c.z.mul_(0.01)
    c.z[torch.arange(4), c.tokens.long()] = torch.tensor([10.0, 15.0, 18.0, 30.0]).cuda()
    c.run()
    ref = c.reference()
    c.check(ref)
    at = (torch.arange(4), c.tokens.cpu().long())
    got, want = R.f64(c.dlogits)[at], ref["dlogits"][0][at]
    # relative: log p = -log(1 + rest) from a sum that is rounded to 2^-24 of 1, so 1 - p is within 2^-23 of itself
    # absolutely
    assert ((got - want).abs() <= 2.0 ** -20 * want.abs() + 2.0 ** -22 * R.f64(c.advantage).abs() * 0.5).all()


def test_offsets_past_2_31_elements():
    rows, gap = 40, 1 << 26
    buf = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda")
    c = Case(rows, 1000, "bf16")
    z, d = (buf.as_strided((rows, 1000), (gap, 1), 2048 * i) for i in range(2))
    z.copy_(c.z)
    s = _seq()
    c.z, c.dlogits = z, d
    c.desc = s.policy_desc(z, d, c.tau, LOW, HIGH, c.kl, 0.5)
    c.run()
    c.check(c.reference())


def test_other_streams_and_graph_replays():
    c = Case(50, 3001, "bf16")
    c.run()
    nan = lambda t: torch.nan_to_num(t.float(), nan=7.0)
    want = [nan(t).clone() for t in (c.loss, c.logp, c.dlogits)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for _ in range(3):
        for t in (c.loss, c.logp, c.dlogits):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((c.loss, c.logp, c.dlogits), want):
            assert torch.equal(nan(t), w)


def test_gradients_against_difference_quotients():
    """fp32: central differences of step e leave (e^2 / 6) times the third derivative, at e = 2^-7 some 1e-4 of the
    advantages and KL terms, and the forward's rounding over e, 2^-22 (|A| + 1) 2^7 a row."""
    c = Case(20, 37, "f32", tau=0.9, masked=False, seed=3)
    c.run()
    e = 2.0 ** -7
    way = torch.randn(c.z.shape, generator=torch.Generator().manual_seed(2)).cuda()
    got = R.f64(c.dlogits * way).sum(1) / (0.5 * R.f64(c.weight))
    keep, ends = c.z.clone(), []
    for sign in (1, -1):
        c.z.copy_(keep + sign * e * way)
        c.run()
        ends.append(R.f64(c.loss))
    slope = (ends[0] - ends[1]) / (2 * e)
    A = R.f64(c.advantage).abs()
    lp = R.f64(c.logp)
    # rows whose ratio crosses a bound between the two ends have a kink there
    ratio = torch.exp(torch.log_softmax(R.f64(keep) / c.tau, 1)[torch.arange(20), c.tokens.cpu().long()] - R.f64(c.old))
    clear = ((ratio - (1 - LOW)).abs() > 0.08) & ((ratio - (1 + HIGH)).abs() > 0.08)
    assert int(clear.sum()) >= 10
    off = (slope - got).abs()
    assert (off[clear] <= (1e-3 * (A + 1) * way.cpu().double().abs().amax(1) ** 3)[clear]).all(), (off / (A + 1))[clear].max()
