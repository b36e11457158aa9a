"""The clipped policy loss on the GPU against its definition in 64 bits (block_ref), elementwise, at the class counts,
strides and masks where its kernel can go wrong; the space around every output stays as it was."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import DT, within
from tests.test_gpu_seq import Framed

pytestmark = pytest.mark.gpu

LOW, HIGH = 0.2, 0.28


def _seq():
    from paper_2103_08802_amd import seq
    return seq


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Case:
    def __init__(self, n, V, dtype, tau=1.0, kl=0.1, old=True, weight=True, lead=0, pad=0, spread=2.0, masked=True, seed=0):
        g = torch.Generator().manual_seed(seed + n + V)
        self.dtype, self.tau, self.kl = dtype, tau, kl
        self.zf = Framed((n, V), DT[dtype], lead, pad, torch.randn(n, V, generator=g) * spread)
        self.z = self.zf.t
        self.tokens = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
        lp = torch.log_softmax(self.z.cpu().double() / tau, 1)[torch.arange(n), self.tokens.long()]
        off = torch.rand(n, generator=g) * 1.2 - 0.6
        for border in (math.log(1 - LOW), math.log(1 + HIGH)):
            off = torch.where((off - border).abs() < 0.01, 0.0, off)
        self.old = (lp - off).float().cuda() if old else None
        self.ref = (lp + 0.5 * torch.randn(n, generator=g)).float().cuda() if kl != 0 else None
        self.advantage = torch.randn(n, generator=g).cuda()
        self.weight = (torch.rand(n, generator=g) + 0.5).cuda() if weight else None
        if masked and n > 4:
            self.tokens[torch.rand(n, generator=g) < 0.2] = -1
            self.tokens[1], self.tokens[2] = -7, V
        self.tokens = self.tokens.cuda()
        self.lf, self.pf = (Framed((1, n), torch.float32, 1) for _ in range(2))
        self.loss, self.logp = self.lf.t[0], self.pf.t[0]
        self.df = Framed((n, V), DT[dtype], lead, pad)
        self.dlogits = self.df.t
        self.desc = _seq().policy_desc(self.z, self.dlogits, tau, LOW, HIGH, kl, 0.5)

    def run(self, dlogits="dlogits", logp="logp"):
        get = lambda n: None if n is None else getattr(self, n)
        _seq().pnn_policy_fwd_bwd(self.desc, self.z, self.tokens, self.advantage, self.old, self.ref, self.weight,
                                  self.loss, get(logp), get(dlogits), _stream())

    def reference(self):
        d = self.desc
        return R.policy(self.z, self.tokens, self.advantage, self.old, self.ref, self.weight, d.temperature, d.clip_low,
                        d.clip_high, d.kl, d.scale)

    def check(self, ref, names=("loss", "logp", "dlogits")):
        for n in names:
            try:
                within(getattr(self, n), *ref[n], self.dtype if n == "dlogits" else "f32")
            except AssertionError as e:
                raise AssertionError(n, *e.args) from None
        for f in (self.zf, self.lf, self.pf, self.df):
            f.intact()


CASES = [
    # n, V, dtype, tau, kl, old, weight, lead, pad
    (1, 1, "f32", 1.0, 0.1, True, False, 0, 0),
    (9, 2, "bf16", 1.0, 0.1, True, True, 0, 0),
    (9, 7, "bf16", 0.7, 0.0, True, True, 1, 2),
    (20, 17, "f32", 1.5, 0.1, False, False, 3, 0),
    (33, 1000, "f32", 1.0, 0.1, True, True, 0, 0),
    (33, 1003, "bf16", 2.0, 0.3, True, True, 0, 0),
    (12, 2048, "bf16", 1.0, 0.1, True, True, 0, 0),
    (12, 2061, "bf16", 1.0, 0.1, True, True, 0, 3),
    (8, 4099, "f32", 0.7, 0.1, True, True, 0, 0),
    (8, 8200, "bf16", 1.0, 0.1, True, True, 0, 0),
    (6, 16391, "f32", 1.0, 0.1, True, False, 1, 1),
    (6, 32771, "bf16", 1.0, 0.1, True, True, 0, 0),
    (6, 65536, "bf16", 1.0, 0.1, True, True, 0, 0),
    (5, 70001, "bf16", 1.0, 0.1, True, True, 0, 0),
    (5, 70001, "f32", 1.0, 0.1, True, True, 0, 0),      # read twice
    (5, 140003, "bf16", 1.0, 0.1, True, True, 0, 0),    # read twice
]


@pytest.mark.parametrize("n,V,dtype,tau,kl,old,weight,lead,pad", CASES)
def test_policy(n, V, dtype, tau, kl, old, weight, lead, pad):
    c = Case(n, V, dtype, tau, kl, old, weight, lead, pad)
    ref = c.reference()
    c.run()
    c.check(ref)
    # without the gradient, without log probabilities, then the gradient in the logits' place
    first = [c.loss.clone(), c.logp.clone(), c.dlogits.clone()]
    c.run(dlogits=None)
    c.run(logp=None)
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=9e9), torch.nan_to_num(b.float(), nan=9e9))
    assert same(c.loss, first[0]) and same(c.logp, first[1]) and same(c.dlogits, first[2])
    c.run(dlogits="z")
    assert same(c.z, first[2])
    c.zf.intact()
