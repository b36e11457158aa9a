"""A small sequence model on the GPU that runs the sequence operators together: trained towards a teacher's top
logits, and answering one token at a time.

    rows = scale table[token]            [x | gate], one row of twice the channels   pnn_embed_fwd
    h_t = f_t h_{t-1} + (1 - f_t) x_t    f = sigmoid(gate)                           pnn_scan_fwd
    logits = h W^T                       a library product
    loss, dL/dlogits                     teacher's top logits and labels             pnn_distill_fwd_bwd
    dL/dh = dL/dlogits W, dL/dW          library products
    dL/dx, dL/dgate                                                                  pnn_scan_bwd
    dL/dtable                            one order of every sum                      pnn_embed_bwd

The recurrence is the evolution the parareal construction splits into intervals, here in time: intervals from a zero
state in parallel, a sequential chain over their ends, a correction of every interval (eqs. (rk) - (tildey)), with a
coarse propagator (the product of an interval's gates) that is exact.

PyTorch supplies device memory, the stream and the plain matrix products; ``python -m paper_2103_08802_amd.seqstep``
trains one on a fixed random teacher and lets it answer.
"""
from __future__ import annotations

import math

from . import seq as Q


class SequenceModel:
    """Device state of the model and its training step for ``batch`` sequences of ``length`` tokens.

    dtype: "bf16" or "f32", the storage type of the parameters, activations and their gradients (the table's gradient
    is float; W's, a library product, is rounded to the storage type).  Tokens below zero are padding; they take part
    in no loss if their labels are below zero and their rows have no teacher entries."""

    def __init__(self, vocab, channels, batch, length, top, dtype="bf16", temperature=2.0, alpha=0.5, seed=0,
                 device="cuda"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("SequenceModel needs a GPU (HIP device)")
        self.torch = torch
        self.vocab, self.channels, self.batch, self.length = vocab, channels, batch, length
        dev = torch.device(device)
        sdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.sdt, self.dev = sdt, dev
        n, D = batch * length, channels
        gen = torch.Generator().manual_seed(seed)
        act = dict(dtype=sdt, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        table = torch.randn(vocab, 2 * D, generator=gen) / math.sqrt(2 * D)
        self.table = table.to(dev).to(sdt)
        self.w = (torch.randn(vocab, D, generator=gen) * math.sqrt(2.0 / D)).to(dev).to(sdt)
        self.scale = math.sqrt(2 * D)
        self.tokens = torch.zeros(batch, length, dtype=torch.int64, device=dev)
        self.labels = torch.zeros(n, dtype=torch.int32, device=dev)
        self.index = torch.zeros(n, top, dtype=torch.int32, device=dev)
        self.teacher = torch.zeros(n, top, **f32)
        self.rows, self.drows = torch.zeros(batch, length, 2 * D, **act), torch.zeros(batch, length, 2 * D, **act)
        self.h, self.dh = torch.zeros(batch, length, D, **act), torch.zeros(batch, length, D, **act)
        self.logits = torch.zeros(n, vocab, **act)          # the gradient takes their place
        self.loss = torch.zeros(n, **f32)
        self.dtable = torch.zeros(vocab, 2 * D, **f32)
        self.x, self.gate = self.rows[..., :D], self.rows[..., D:]
        self.dx, self.dgate = self.drows[..., :D], self.drows[..., D:]
        self.embed = Q.embed_desc(self.table, self.tokens, self.rows.view(n, 2 * D), self.scale)
        self.scan = Q.scan_desc(self.x, self.gate, self.h, self.dh, self.dx, self.dgate)
        self.distill = Q.distill_desc(self.logits, self.teacher, self.logits, temperature, alpha, 1.0 / n)
        states, ws = Q.pnn_scan_sizes(self.scan)
        self.states = torch.zeros(max(states // 4, 1), **f32)
        self.ws = torch.zeros(max(ws, Q.pnn_embed_workspace_size(self.embed), 256), dtype=torch.uint8, device=dev)
        # answering: one token of every sequence, its state in place
        self.token1 = torch.zeros(batch, dtype=torch.int64, device=dev)
        self.rows1 = torch.zeros(batch, 1, 2 * D, **act)
        self.h1 = torch.zeros(batch, 1, D, **act)
        self.state = torch.zeros(batch, D, **f32)
        self.embed1 = Q.embed_desc(self.table, self.token1, self.rows1.view(batch, 2 * D), self.scale)
        self.scan1 = Q.scan_desc(self.rows1[..., :D], self.rows1[..., D:], self.h1)

    def stream(self):
        return self.torch.cuda.current_stream(self.dev).cuda_stream

    def load(self, tokens, index, teacher, labels):
        """tokens [batch][length]; per token: the teacher's classes and logits [top] and the label (below 0: none)."""
        self.tokens.copy_(tokens.view_as(self.tokens))
        self.index.copy_(index.view_as(self.index))
        self.teacher.copy_(teacher.view_as(self.teacher))
        self.labels.copy_(labels.view_as(self.labels))

    def forward(self, lengths=None, state=None, keep=True):
        """The states h of the loaded tokens, and the states after the last step (self.state).  ``lengths``: int32,
        the tokens of each sequence that count; ``state``: the states to start from (None: zero)."""
        s = self.stream()
        Q.pnn_embed_fwd(self.embed, self.table, self.tokens, self.rows, s)
        Q.pnn_scan_fwd(self.scan, self.x, self.gate, lengths, state, self.h, self.state,
                       self.states if keep else None, self.ws, s)

    def step(self, lengths=None):
        """Forward, loss and gradients: self.loss [batch * length], self.dtable, and dW as the result."""
        t, s = self.torch, self.stream()
        self.forward(lengths)
        h = self.h.view(-1, self.channels)
        t.mm(h, self.w.t(), out=self.logits)
        Q.pnn_distill_fwd_bwd(self.distill, self.logits, self.index, self.teacher, self.labels, None, self.loss,
                              self.logits, s)
        t.mm(self.logits, self.w, out=self.dh.view(-1, self.channels))
        dw = t.mm(self.logits.t(), h)
        Q.pnn_scan_bwd(self.scan, self.x, self.gate, lengths, self.states, self.dh, None, self.dx, self.dgate, None,
                       self.ws, s)
        Q.pnn_embed_bwd(self.embed, self.drows, self.tokens, self.dtable, False, self.ws, s)
        return dw

    def update(self, dw, lr):
        """Plain gradient descent on both parameters."""
        self.table.add_(self.dtable.to(self.sdt), alpha=-lr)
        self.w.add_(dw.to(self.sdt), alpha=-lr)

    def answer_step(self):
        """One token of every sequence (self.token1): the next one by the largest logit, in its place.  Nothing here
        looks at the host, so the step can be captured into a graph."""
        s = self.stream()
        Q.pnn_embed_fwd(self.embed1, self.table, self.token1, self.rows1, s)
        Q.pnn_scan_fwd(self.scan1, self.rows1[..., :self.channels], self.rows1[..., self.channels:], None, self.state,
                       self.h1, self.state, None, None, s)
        logits = self.torch.mm(self.h1[:, 0], self.w.t())
        self.token1.copy_(logits.argmax(1))

    def answer(self, tokens, steps):
        """Continues prompts [batch][length] by ``steps`` tokens, one at a time from the prompts' states."""
        t = self.torch
        self.tokens.copy_(tokens.view_as(self.tokens))
        self.forward(keep=False)
        self.token1.copy_(t.mm(self.h[:, -1], self.w.t()).argmax(1))
        out = t.empty(self.batch, steps, dtype=t.int64, device=self.dev)
        for i in range(steps):
            if i > 0:
                self.answer_step()
            out[:, i] = self.token1
        return out


def main():
    import torch
    vocab, channels, batch, length, top = 4096, 256, 8, 512, 16
    m = SequenceModel(vocab, channels, batch, length, top)
    g = torch.Generator().manual_seed(1)
    tokens = torch.randint(0, vocab, (batch, length), generator=g)
    index = torch.stack([torch.randperm(vocab, generator=g)[:top] for _ in range(vocab)])[tokens]   # by the token
    teacher = torch.randn(batch, length, top, generator=g) * 2
    m.load(tokens, index, teacher, index[..., 0])
    for i in range(50):
        dw = m.step()
        m.update(dw, 2.0)
        if i % 10 == 0 or i == 49:
            print(f"step {i:3d}  loss {m.loss.mean().item():.4f}", flush=True)
    print("answer", m.answer(tokens, 8)[0].tolist(), flush=True)


if __name__ == "__main__":
    main()
