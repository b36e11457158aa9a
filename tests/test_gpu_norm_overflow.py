"""Rows whose squares pass the float range are normed to zeros, with no gradient through that norm."""
import pytest
import torch

from tests.test_gpu_norm import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [24, 2048, 5000])
def test_rows_past_the_float_range(dtype, width):
    clean, c = (Case(6, 1, width, dtype, "pgrnwd", seed=5) for _ in range(2))
    for t in (c.x, c.res):
        t[2] = 2e37                              # sums of dy h and of their squares are infinite
    c.dy[2] = 1.0
    for k in (clean, c):
        k.forward()
        k.backward()
    assert not c.y[2].any()
    assert torch.equal(c.dres[2], c.dh[2]) and not c.dx[2].any() and not c.dgate[2].any()
    assert torch.isfinite(c.f1.t).all() and torch.isfinite(c.f2.t).all()
    rows = [0, 1, 3, 4, 5]
    for n in ("h", "y", "dx", "dgate", "dres"):
        assert torch.equal(getattr(clean, n)[rows], getattr(c, n)[rows])
