"""What the block model takes its inputs from: a batch's own, never the one's before it or its padding's."""
import pytest
import torch

from tests.test_gpu_blockstep import _loaded, _model

pytestmark = pytest.mark.gpu


def test_a_batch_without_advantages_has_not_the_last_ones():
    m, tokens, answers, *_ = _loaded()
    fresh = _model()
    for one in (m, fresh):
        one.load(tokens.cuda(), answers.cuda())
    got, want = m.step(), fresh.step()
    assert torch.equal(m.loss, fresh.loss) and torch.equal(m.dtable, fresh.dtable)
    assert all(torch.equal(got[k], want[k]) for k in want)
