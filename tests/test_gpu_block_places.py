"""Tensors that a call does not look at may stand anywhere, an output's place included, and the states in one another's."""
import pytest
import torch

from tests.test_gpu_linattn import Case as Linattn
from tests.test_gpu_norm import Case as Norm
from tests.test_gpu_linattn import _seq, _stream

pytestmark = pytest.mark.gpu


def test_a_workspace_of_no_bytes():
    c = Linattn(2, 40, 2, 2, 16, 24, "bf16")
    s = _seq()
    assert s.pnn_linattn_sizes(c.desc)[0] == 0
    c.forward()
    want = c.o.clone(), c.sT.clone()
    o = torch.zeros(c.o.shape, dtype=c.o.dtype, device="cuda")
    desc = s.linattn_desc(c.q, c.k, c.v, o, scale=c.scale)
    s.pnn_linattn_fwd(desc, c.q, c.k, c.v, c.decay, None, c.s0, o, c.s0, o, _stream())
    assert torch.equal(o, want[0]) and torch.equal(c.s0, want[1])


def test_weights_of_a_norm_left_out():
    c = Norm(20, 1, 64, "f32", "rnw")
    c.forward()
    want = c.h.clone(), c.y.clone()
    s = _seq()
    s.pnn_norm_fwd(c.desc, c.x, c.h, None, c.res, c.w2, c.h, c.y, _stream())
    assert torch.equal(c.h, want[0]) and torch.equal(c.y, want[1])


def test_a_workspace_without_weight_gradients():
    c = Norm(20, 1, 64, "f32", "prnwd")
    c.forward()
    c.backward()
    want = c.dx.clone()
    dx = torch.zeros(c.dx.shape, device="cuda")
    s = _seq()
    desc = s.norm_desc(c.x, res=c.res, dy=c.dy, dh=c.dh, dx=dx, post=True, pre=True, eps=c.desc.eps, alpha=c.alpha)
    s.pnn_norm_bwd(desc, c.x, c.w1, None, c.res, c.w2, c.dy, c.dh, dx, None, None, None, None, False, dx, _stream())
    assert torch.equal(dx, want)
