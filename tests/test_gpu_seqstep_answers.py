"""The number of tokens that the sequence model answers with, none included."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [0, 1, 3])
def test_as_many_answers_as_asked_for(steps):
    from paper_2103_08802_amd.seqstep import SequenceModel
    m = SequenceModel(37, 24, 3, 21, 5, "f32", seed=4)
    tokens = torch.randint(0, 37, (3, 21), generator=torch.Generator().manual_seed(8)).cuda()
    got = m.answer(tokens, steps)
    assert got.shape == (3, steps) and got.dtype == torch.int64
    assert torch.equal(got, m.answer(tokens, 4)[:, :steps])
