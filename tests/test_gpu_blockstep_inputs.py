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


def test_answers_to_empty_prompts_do_not_depend_on_padding():
    m = _model()
    g = torch.Generator().manual_seed(7)
    tokens = torch.randint(0, m.vocab, (m.batch, m.length), generator=g)
    other = torch.randint(0, m.vocab, (m.batch, m.length), generator=g)
    lengths = torch.tensor([0, 9, -2], dtype=torch.int32)
    other[1, :9] = tokens[1, :9]
    noise = -torch.log(-torch.log(torch.rand(4, m.batch, m.vocab, generator=g))).cuda()
    got = m.answer(tokens.cuda(), noise, lengths.cuda())
    assert torch.equal(got, m.answer(other.cuda(), noise, lengths.cuda()))
    # no logits: the noise alone draws, and the answers go on from a state of zeros
    assert torch.equal(got[[0, 2], 0], noise[0, [0, 2]].argmax(1))
    one = _model(length=1)
    after = one.answer(got[:, :1], noise[1:])
    assert torch.equal(got[[0, 2], 1:], after[[0, 2]])
