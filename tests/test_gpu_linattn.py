"""Linear attention on the GPU against its definition in 64 bits (block_ref), elementwise, at the lengths, widths, head
layouts, masks and strides where its kernels can go wrong; the space around every output stays as it was."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import DT, within
from tests.test_gpu_seq import Framed

pytestmark = pytest.mark.gpu


def _seq():
    from paper_2103_08802_amd import seq
    return seq


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _ws(bytes_):
    return torch.full((max(bytes_, 256),), 0xCD, dtype=torch.uint8, device="cuda")


class Case:
    """Inputs and framed outputs of a call.  layout: "steps" [batch][length][heads][width], "heads"
    [batch][heads][length][width], "time" [length][batch][heads][width]; lead, pad: see Framed."""

    def __init__(self, B, T, H, kv, K, V, dtype, layout="steps", ragged=False, state=True, lead=0, pad=0, seed=0):
        g = torch.Generator().manual_seed(seed + 31 * T + K + V)
        self.args = (B, T, H, kv, K, V)
        self.dtype, self.layout, self.lead, self.pad = dtype, layout, lead, pad
        self.g = g
        self.scale = 0.3
        self.frames = {}
        for n, h, w in (("q", H, K), ("k", kv, K), ("v", kv, V), ("dout", H, V)):
            setattr(self, n, self.tensor(n, h, w, torch.randn(B, T, h, w, generator=g)))
        for n, h, w in (("o", H, V), ("dq", H, K), ("dk", kv, K), ("dv", kv, V)):
            setattr(self, n, self.tensor(n, h, w))
        self.decay = -torch.exp2(-4 * torch.rand(H, generator=g) - 1).cuda()
        self.lengths = None
        if ragged:
            self.lengths = torch.randint(-2, T + 3, (B,), generator=g, dtype=torch.int32)
            self.lengths[0] = T
            if B > 1:
                self.lengths[-1] = 0
            self.lengths = self.lengths.cuda()
        f = lambda n: Framed((B, H, K, V), torch.float32, 1, 0, n)
        self.fs = {n: f(torch.randn(B, H, K, V, generator=g)) for n in ("s0", "dsT")}
        self.fs.update({n: f(None) for n in ("sT", "ds0")})
        for n in ("s0", "dsT", "sT", "ds0"):
            setattr(self, n, self.fs[n].t if state else None)
        s = _seq()
        self.desc = s.linattn_desc(self.q, self.k, self.v, self.o, self.dout, self.dq, self.dk, self.dv, self.scale)

    def tensor(self, name, h, w, fill=None):
        B, T = self.args[:2]
        order = {"steps": (0, 1, 2), "heads": (0, 2, 1), "time": (1, 0, 2)}[self.layout]
        dims = (B, T, h)
        f = Framed([dims[i] for i in order] + [w], DT[self.dtype], self.lead, self.pad)
        self.frames[name] = f
        t = f.t.permute(*[order.index(i) for i in range(3)], 3)
        if fill is not None:
            t.copy_(fill)
        return t

    def forward(self, s0="s0", sT="sT"):
        s = _seq()
        s.pnn_linattn_fwd(self.desc, self.q, self.k, self.v, self.decay, self.lengths, getattr(self, s0), self.o,
                          getattr(self, sT), _ws(s.pnn_linattn_sizes(self.desc)[0]), _stream())

    def backward(self):
        s = _seq()
        s.pnn_linattn_bwd(self.desc, self.q, self.k, self.v, self.decay, self.lengths, self.s0, self.dout, self.dsT,
                          self.dq, self.dk, self.dv, self.ds0, _ws(s.pnn_linattn_sizes(self.desc)[1]), _stream())

    def reference(self, backward=True):
        return R.linattn(self.q, self.k, self.v, self.decay, self.lengths, self.s0, self.desc.scale, self.dtype,
                         self.dout if backward else None, self.dsT)

    def check(self, ref):
        for n, (value, bound) in ref.items():
            got = getattr(self, n)
            if got is None:
                continue
            try:
                within(got, value, bound, "f32" if n in ("sT", "ds0") else self.dtype)
            except AssertionError as e:
                raise AssertionError(n, *e.args) from None
        for f in list(self.frames.values()) + list(self.fs.values()):
            f.intact()


CASES = [
    # B, T, H, kv, K, V, dtype, layout, ragged, state, lead, pad
    (1, 1, 1, 1, 1, 1, "f32", "steps", False, True, 0, 0),
    (1, 2, 1, 1, 8, 8, "bf16", "steps", False, False, 0, 0),
    (2, 15, 2, 1, 16, 17, "bf16", "steps", False, True, 1, 1),
    (2, 16, 2, 2, 7, 5, "f32", "heads", True, True, 3, 2),
    (3, 17, 3, 1, 33, 64, "bf16", "time", True, True, 0, 0),
    (2, 31, 4, 2, 64, 65, "f32", "steps", True, False, 0, 4),
    (1, 63, 2, 2, 64, 64, "bf16", "heads", False, True, 0, 0),
    (1, 64, 2, 1, 65, 128, "bf16", "steps", False, True, 8, 8),
    (2, 65, 2, 2, 128, 128, "bf16", "steps", True, True, 0, 0),
    (2, 127, 3, 3, 40, 72, "f32", "time", True, True, 1, 0),
    (1, 128, 1, 1, 129, 130, "bf16", "steps", False, True, 0, 0),
    (2, 129, 2, 1, 200, 256, "bf16", "heads", True, True, 2, 6),
    (1, 100, 2, 2, 256, 40, "f32", "steps", False, True, 0, 0),
    (1, 97, 2, 2, 24, 256, "f32", "steps", False, False, 0, 0),
    (4, 300, 6, 2, 48, 80, "bf16", "steps", True, True, 0, 0),         # segments
    (1, 1030, 2, 1, 64, 96, "bf16", "steps", False, True, 0, 0),       # many segments
    (2, 700, 2, 2, 128, 64, "f32", "heads", True, True, 0, 0),
    (40, 70, 8, 8, 16, 16, "bf16", "steps", True, True, 0, 0),         # one segment: enough heads
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_linattn(case):
    c = Case(*case)
    c.forward()
    c.backward()
    c.check(c.reference())
    # the same bits again, and from another workspace's contents
    names = [n for n in ("o", "sT", "dq", "dk", "dv", "ds0") if getattr(c, n) is not None]
    first = [getattr(c, n).clone() for n in names]
    c.forward()
    c.backward()
    for n, t in zip(names, first):
        assert torch.equal(getattr(c, n), t), n
