"""The sequence model's training step against 64-bit autograd, and its answers step by step against whole sequences."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _model(dtype="f32", vocab=37, channels=24, batch=3, length=21, top=5):
    from paper_2103_08802_amd.seqstep import SequenceModel
    m = SequenceModel(vocab, channels, batch, length, top, dtype, 2.0, 0.5, seed=4)
    g = torch.Generator().manual_seed(8)
    tokens = torch.randint(0, vocab, (batch, length), generator=g)
    tokens[0, 3] = -1
    index = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(batch * length)])
    teacher = torch.randn(batch * length, top, generator=g)
    labels = torch.randint(0, vocab, (batch * length,), generator=g)
    labels[5:9], index[5:7] = -1, -1
    m.load(tokens, index, teacher, labels)
    return m, tokens, index, teacher, labels


def _loss(table, w, scale, tokens, index, teacher, labels, tau, alpha, lengths=None):
    B, T = tokens.shape
    D = w.shape[1]
    rows = torch.where((tokens >= 0)[..., None], table[tokens.clamp(min=0)] * scale, 0.0)
    h, out = torch.zeros(B, D, dtype=torch.float64), []
    for t in range(T):
        f = torch.sigmoid(rows[:, t, D:])
        new = f * h + (1 - f) * rows[:, t, :D]
        live = torch.ones(B, 1, dtype=torch.bool) if lengths is None else (t < lengths)[:, None]
        h = torch.where(live, new, h)
        out.append(torch.where(live, h, 0.0))
    z = torch.stack(out, 1).reshape(B * T, D) @ w.t()
    held = index >= 0
    p = torch.softmax((teacher.double() / tau).masked_fill(~held, -1e30), 1) * held
    logq = torch.log_softmax(z / tau, 1).gather(1, index.clamp(min=0).long())
    kl = torch.where(p > 0, p * (torch.log(p.clamp(min=1e-300)) - logq), 0.0).sum(1)
    ce = -torch.log_softmax(z, 1).gather(1, labels.clamp(min=0).long()[:, None])[:, 0] * (labels >= 0)
    return alpha * tau ** 2 * kl + (1 - alpha) * ce


@pytest.mark.parametrize("ragged", [False, True])
def test_training_step_gradients(ragged):
    """fp32: sums of at most 37 (vocabulary) x 24 x 63 terms of like size, 2^-24 each, through 21 steps: 1e-5 of the
    largest gradient."""
    m, tokens, index, teacher, labels = _model()
    lengths = torch.tensor([21, 0, 13], dtype=torch.int32) if ragged else None
    dw = m.step(None if lengths is None else lengths.cuda())
    table, w = m.table.cpu().double().requires_grad_(), m.w.cpu().double().requires_grad_()
    loss = _loss(table, w, m.embed.scale, tokens, index, teacher, labels, 2.0, 0.5, lengths)
    loss.mean().backward()
    near = lambda a, b: (a.cpu().double() - b).abs().max() <= 1e-5 * b.abs().max()
    assert near(m.loss, loss.detach())
    assert near(m.dtable, table.grad) and near(dw, w.grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_lowers_the_loss(dtype):
    m, *_ = _model(dtype)
    losses = []
    for _ in range(30):
        dw = m.step()
        losses.append(m.loss.mean().item())
        m.update(dw, 1.0)
    assert losses[-1] < 0.8 * losses[0], losses


def test_answers_step_by_step_are_those_of_the_whole_sequence():
    m, tokens, *_ = _model()
    tokens = tokens.clamp(min=0).cuda()
    got = m.answer(tokens, 4)
    seq = tokens
    from paper_2103_08802_amd.seqstep import SequenceModel
    for i in range(4):
        w = SequenceModel(m.vocab, m.channels, m.batch, seq.shape[1], 5, "f32", seed=4)
        w.tokens.copy_(seq)
        w.forward(keep=False)
        z = torch.mm(w.h[:, -1], w.w.t())
        top = z.topk(2, 1)
        clear = top.values[:, 0] - top.values[:, 1] > 1e-3      # ties by rounding are nobody's mistake
        assert torch.equal(got[clear, i], top.indices[clear, 0])
        seq = torch.cat([seq, got[:, i:i + 1]], 1)


def test_answer_step_in_a_graph():
    m, tokens, *_ = _model("bf16")
    tokens = tokens.clamp(min=0).cuda()
    want = m.answer(tokens, 5)
    m.answer(tokens, 1)                          # the prompt's states and first answer, as captured below
    first, state = m.token1.clone(), m.state.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.answer_step()
    for _ in range(2):
        m.token1.copy_(first)
        m.state.copy_(state)
        got = [first]
        for _ in range(4):
            g.replay()
            got.append(m.token1.clone())
        assert torch.equal(torch.stack(got, 1), want)
