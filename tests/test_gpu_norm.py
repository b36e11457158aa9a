"""Norms around a block on the GPU against their definition in 64 bits (block_ref), elementwise, at the widths, strides
and combinations of parts where the kernels can go wrong; the space around every output stays as it was."""
import math

import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import DT, within
from tests.test_gpu_seq import Framed

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _seq():
    from paper_2103_08802_amd import seq
    return seq


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _checked(name, got, ref, dtype):
    try:
        within(got, *ref, dtype)
    except AssertionError as e:
        raise AssertionError(name, *e.args) from None


class Case:
    def __init__(self, rows, heads, width, dtype, parts, lead=0, pad=0, swap=False, seed=0, spread=1.0):
        """parts: letters of p(ost), g(ate), r(es), n (norm before the next block), w(eights), d(h); swap: heads outside
        rows"""
        g = torch.Generator().manual_seed(seed + rows + 7 * width)
        self.dtype = dtype
        self.post, self.pre = "p" in parts, "n" in parts
        dims = (heads, rows, width) if swap else (rows, heads, width)
        self.frames = {}

        def tensor(name, on, fill):
            t = None
            if on:
                f = Framed(dims, DT[dtype], lead, pad, torch.randn(dims, generator=g) * spread if fill else None)
                self.frames[name] = f
                t = f.t.transpose(0, 1) if swap else f.t
            setattr(self, name, t)

        tensor("x", True, True)
        tensor("gate", "g" in parts, True)
        tensor("res", "r" in parts, True)
        tensor("dy", self.pre, True)
        tensor("dh", "d" in parts, True)
        for n in ("h", "dx", "dres"):
            tensor(n, True, False)
        tensor("y", self.pre, False)
        tensor("dgate", "g" in parts, False)
        weight = lambda on: 1 + 0.3 * torch.randn(width, generator=g) if on and "w" in parts else None
        self.w_post, self.w_pre = weight(self.post), weight(self.pre)
        cuda = lambda w: None if w is None else w.cuda()
        self.w1, self.w2 = cuda(self.w_post), cuda(self.w_pre)
        old = lambda on: Framed((1, width), torch.float32, 1, 0, torch.randn(1, width, generator=g)) if on else None
        self.f1, self.f2 = old(self.post), old(self.pre)
        self.alpha = 0.75
        self.width = width
        s = _seq()
        self.desc = s.norm_desc(self.x, gate=self.gate, res=self.res, h=self.h, y=self.y, dy=self.dy, dh=self.dh,
                                dx=self.dx, dgate=self.dgate, dres=self.dres, post=self.post, pre=self.pre, eps=EPS,
                                alpha=self.alpha)

    def forward(self):
        _seq().pnn_norm_fwd(self.desc, self.x, self.w1, self.gate, self.res, self.w2, self.h, self.y, _stream())

    def backward(self, accumulate=False, dres="dres"):
        s = _seq()
        ws = torch.full((max(s.pnn_norm_workspace_size(self.desc), 256),), 0xCD, dtype=torch.uint8, device="cuda")
        one = lambda f: None if f is None else f.t[0]
        s.pnn_norm_bwd(self.desc, self.x, self.w1, self.gate, self.res, self.w2, self.dy, self.dh, self.dx, self.dgate,
                       getattr(self, dres), one(self.f1), one(self.f2), accumulate, ws, _stream())

    def check_forward(self):
        ref = R.norm_fwd(self.x, self.w_post, self.gate, self.res, self.w_pre, self.post, self.pre, self.desc.eps,
                         self.alpha)
        for n, v in ref.items():
            _checked(n, getattr(self, n), v, self.dtype)
        self.intact()

    def reference(self):
        return R.norm_bwd(self.x, self.w_post, self.gate, self.res, self.w_pre, self.dy, self.dh, self.post, self.pre,
                          self.desc.eps, self.alpha)

    def check_backward(self, ref, first=None):
        for n, v in ref.items():
            if n in ("dw_post", "dw_pre"):
                f = self.f1 if n == "dw_post" else self.f2
                if first is not None:
                    v = (v[0] + first[n], v[1] + 2 * R.U * (v[0].abs() + first[n].abs()))
                _checked(n, f.t[0], v, "f32")
            else:
                _checked(n, getattr(self, n), v, self.dtype)
        self.intact()

    def intact(self):
        for f in list(self.frames.values()) + [f for f in (self.f1, self.f2) if f is not None]:
            f.intact()


CASES = [
    # rows, heads, width, dtype, parts, lead, pad, swap
    (1, 1, 1, "f32", "pgrnwd", 0, 0, False),
    (3, 1, 8, "bf16", "n", 0, 0, False),
    (5, 1, 7, "bf16", "pgrnwd", 1, 2, False),
    (33, 3, 16, "f32", "pg", 0, 4, True),
    (70, 2, 64, "f32", "prnw", 3, 1, False),
    (65, 4, 100, "f32", "grd", 0, 0, True),
    (65, 5, 128, "bf16", "pgwd", 0, 0, False),
    (40, 2, 129, "bf16", "pgrnwd", 5, 0, False),
    (17, 1, 256, "f32", "pgrnwd", 0, 0, False),
    (19, 1, 257, "bf16", "rnwd", 0, 0, False),
    (9, 2, 512, "bf16", "pn", 8, 8, False),
    (9, 1, 515, "f32", "pgrnwd", 0, 0, False),
    (30, 1, 1000, "bf16", "pgrnwd", 0, 0, False),
    (6, 1, 1030, "f32", "pnwd", 1, 0, False),
    (4, 1, 2048, "bf16", "prnwd", 0, 0, False),
    (3, 1, 2050, "f32", "pgrnwd", 0, 0, False),
    (5, 1, 4096, "bf16", "pgrnwd", 0, 0, False),
    (3, 1, 4100, "f32", "rnwd", 0, 0, False),
    (2, 1, 8191, "bf16", "pgrnwd", 2, 1, False),
    (2, 1, 8200, "f32", "pgrnwd", 0, 0, False),
    (3, 1, 16384, "bf16", "pgrnwd", 0, 0, False),
    (2, 1, 16383, "f32", "pgrnwd", 0, 0, False),
    (2500, 1, 24, "f32", "pgrnwd", 0, 0, False),       # teams walk over several rows
    (700, 31, 16, "bf16", "pgrnwd", 0, 0, True),
    (1100, 1, 2056, "bf16", "pgrnwd", 0, 0, False),    # workgroups walk over several rows
    (300, 1, 4104, "bf16", "pgrnwd", 0, 0, False),
]


@pytest.mark.parametrize("rows,heads,width,dtype,parts,lead,pad,swap", CASES)
def test_norm(rows, heads, width, dtype, parts, lead, pad, swap):
    c = Case(rows, heads, width, dtype, parts, lead, pad, swap)
    c.forward()
    c.check_forward()
    c.backward()
    ref = c.reference()
    c.check_backward(ref)
    names = {"dw_post": c.f1, "dw_pre": c.f2}
    first = {n: f.t[0].cpu().double() for n, f in names.items() if f is not None}
    c.backward(accumulate=True)
    c.check_backward(ref, first)
    # the same bits again, and the residual's gradient in the place of the sum's
    c.backward()
    for n, t in first.items():
        assert torch.equal(names[n].t[0].cpu().double(), t)
    if "d" in parts:
        want = c.dres.clone()
        c.desc.dres = c.desc.dh
        c.backward(dres="dh")
        assert torch.equal(c.dh, want)
