"""Ratios past the float range: an advantage of 0 has no policy term whatever the ratio, a positive one is clipped."""
import pytest
import torch

from tests import block_ref as R
from tests.test_gpu_policy import HIGH, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_ratios_past_the_float_range(dtype, kl):
    c = Case(4, 300, dtype, kl=kl, masked=False)
    lp = torch.log_softmax(R.f64(c.z) / c.tau, 1)[torch.arange(4), c.tokens.cpu().long()]
    c.old.copy_((lp - torch.tensor([100.0, 100.0, 95.0, 0.05])).float())
    c.advantage.copy_(torch.tensor([0.0, 2.0, -0.0, 0.0]))
    c.run()
    c.check(c.reference())
    if kl == 0:
        assert not c.dlogits.any() and c.loss[1] == -torch.tensor(1 + HIGH, dtype=torch.float32) * 2
        assert not c.loss[[0, 2, 3]].any()


def test_logits_that_are_not_finite_stay_so_without_an_advantage():
    c = Case(3, 300, "f32", kl=0.0, masked=False)
    c.advantage.zero_()
    c.z[1, 7] = float("nan")
    c.run()
    assert torch.isnan(c.loss[1]) and torch.isnan(c.dlogits[1]).all() and not c.loss[[0, 2]].any()
