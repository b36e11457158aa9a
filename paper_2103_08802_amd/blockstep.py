"""A sequence model of residual blocks on the GPU, trained by its own answers: linear attention with a decay for each
head between norms, and the clipped policy loss.

    h = table[token] sqrt(D)                                           pnn_embed_fwd
    y = w norm(h)                                                      pnn_norm_fwd
    every block:
        [q | k | v | g] = y Win^T                                      a library product
        o_t = q_t S_t / sqrt(dk),  S_t = lambda S_{t-1} + k_t v_t^T    pnn_linattn_fwd
        a = w norm(o) silu(g), head by head                            pnn_norm_fwd
        b = a Wout^T                                                   a library product
        h <- h + alpha b,  y = w norm(h)                               pnn_norm_fwd
    logits = y W^T                                                     a library product
    loss, dL/dlogits                                                   pnn_policy_fwd_bwd
and the way back by the _bwd entry points.

PyTorch supplies device memory, the stream, the plain matrix products and the drawing of tokens; ``python -m
paper_2103_08802_amd.blockstep`` lets one answer, and trains it to answer with even tokens.
"""
from __future__ import annotations

import math

from . import seq as Q


class BlockModel:
    """Device state of the model and its training step for ``batch`` sequences of ``length`` tokens.

    dtype: "bf16" or "f32", the storage type of the parameters, activations and their gradients (norm weights and their
    gradients, and the table's gradient, are float).  Tokens below zero are padding: they enter as zeros."""

    EPS = 1e-5

    def __init__(self, vocab, width, heads, key_width, value_width, blocks, batch, length, dtype="bf16", temperature=1.0,
                 clip=0.2, kl=0.02, seed=0, device="cuda"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("BlockModel needs a GPU (HIP device)")
        if blocks < 1:
            raise ValueError("a model has at least one block")
        self.torch = torch
        self.vocab, self.batch, self.length, self.blocks = vocab, batch, length, blocks
        self.dev = dev = torch.device(device)
        self.sdt = sdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        D, H, K, V, n = width, heads, key_width, value_width, batch * length
        self.D, self.H, self.K, self.V, self.n = D, H, K, V, n
        self.temperature = temperature
        gen = torch.Generator().manual_seed(seed)
        weight = lambda *s: (torch.randn(*s, generator=gen) / math.sqrt(s[1])).to(dev).to(sdt)
        self.table = (torch.randn(vocab, D, generator=gen) / math.sqrt(D)).to(dev).to(sdt)
        P = H * (2 * K + 2 * V)
        ones = lambda w: torch.ones(w, device=dev)
        self.layers = [{"win": weight(P, D), "wout": weight(D, H * V), "wo": ones(V), "wy": ones(D)} for _ in range(blocks)]
        self.wy0, self.w = ones(D), weight(vocab, D)
        self.alpha = 1.0 / math.sqrt(blocks)
        # heads that keep a token for 8 to 1024 steps
        self.decay = (-torch.exp2(-3 - 7 * (torch.arange(H) + 0.5) / H)).to(dev)
        self.whole = self._rows(batch, length)
        self.one = self._rows(batch, 1)
        self.states = [torch.zeros(batch, H, K, V, device=dev) for _ in range(blocks)]
        f32 = dict(dtype=torch.float32, device=dev)
        self.tokens = torch.zeros(batch, length, dtype=torch.int64, device=dev)
        self.answers = torch.full((n,), -1, dtype=torch.int32, device=dev)
        self.advantage, self.old, self.ref = (torch.zeros(n, **f32) for _ in range(3))
        self.loss, self.logp = torch.zeros(n, **f32), torch.zeros(n, **f32)
        self.logits = torch.zeros(n, vocab, dtype=sdt, device=dev)          # the gradient takes their place
        self.policy = Q.policy_desc(self.logits, self.logits, temperature, clip, clip, kl, 1.0 / n)
        self.dtable = torch.zeros(vocab, D, **f32)
        self.embed = Q.embed_desc(self.table, self.tokens, self.whole["h"][0], math.sqrt(D))
        self.token1 = torch.zeros(batch, dtype=torch.int64, device=dev)
        self.embed1 = Q.embed_desc(self.table, self.token1, self.one["h"][0], math.sqrt(D))
        ws = max([Q.pnn_embed_workspace_size(self.embed), 256] +
                 [Q.pnn_norm_workspace_size(self.whole[k]) for k in ("first", "sum", "out")] +
                 list(Q.pnn_linattn_sizes(self.whole["attn"])) + list(Q.pnn_linattn_sizes(self.one["attn"])))
        self.ws = torch.zeros(ws, dtype=torch.uint8, device=dev)

    def _rows(self, batch, length):
        """Activations, their gradients and descriptions for batch x length tokens."""
        t, D, H, K, V, n = self.torch, self.D, self.H, self.K, self.V, batch * length
        new = lambda *s: t.zeros(*s, dtype=self.sdt, device=self.dev)
        r = {"h": [new(n, D) for _ in range(self.blocks + 1)], "y": [new(n, D) for _ in range(self.blocks + 1)]}
        P = H * (2 * K + 2 * V)
        r["p"] = [new(batch, length, P) for _ in range(self.blocks)]
        r["o"], r["a"] = ([new(batch, length, H, V) for _ in range(self.blocks)] for _ in range(2))
        r["b"] = [new(n, D) for _ in range(self.blocks)]
        r["dp"], r["do"], r["da"] = new(batch, length, P), new(batch, length, H, V), new(batch, length, H, V)
        r["dy"], r["dh"], r["db"] = new(n, D), new(n, D), new(n, D)
        q, k, v, g = self.split(r["p"][0])
        dq, dk, dv, dg = self.split(r["dp"])
        r["attn"] = Q.linattn_desc(q, k, v, r["o"][0], r["do"], dq, dk, dv, scale=1.0 / math.sqrt(K))
        rows = lambda x: x.flatten(0, 1)
        r["out"] = Q.norm_desc(rows(r["o"][0]), gate=rows(g), h=rows(r["a"][0]), dh=rows(r["da"]), dx=rows(r["do"]),
                               dgate=rows(dg), post=True, eps=self.EPS)
        h, y, b = r["h"][0], r["y"][0], r["b"][0]
        r["first"] = Q.norm_desc(h, y=y, dy=r["dy"], dh=r["dh"], dx=r["db"], pre=True, eps=self.EPS)
        r["sum"] = Q.norm_desc(b, res=h, h=h, y=y, dy=r["dy"], dh=r["dh"], dx=r["db"], dres=r["dh"], pre=True,
                               eps=self.EPS, alpha=self.alpha, stored=False)
        return r

    def split(self, p):
        """Queries, keys, values and gates [batch][length][heads][width] of the projection's rows."""
        H, K, V = self.H, self.K, self.V
        return [x.unflatten(2, (H, -1)) for x in p.split([H * K, H * K, H * V, H * V], 2)]

    def stream(self):
        return self.torch.cuda.current_stream(self.dev).cuda_stream

    def _forward(self, r, embed, tokens, states, keep, lengths=None):
        """r["y"][-1] of the tokens.  states: those before the first step (None: zero), keep: those after the last."""
        t, s = self.torch, self.stream()
        n = r["h"][0].shape[0]
        Q.pnn_embed_fwd(embed, self.table, tokens, r["h"][0], s)
        Q.pnn_norm_fwd(r["first"], r["h"][0], None, None, None, self.wy0, None, r["y"][0], s)
        for i, w in enumerate(self.layers):
            t.mm(r["y"][i], w["win"].t(), out=r["p"][i].view(n, -1))
            q, k, v, g = self.split(r["p"][i])
            Q.pnn_linattn_fwd(r["attn"], q, k, v, self.decay, lengths, states and states[i], r["o"][i], keep and keep[i],
                              self.ws, s)
            Q.pnn_norm_fwd(r["out"], r["o"][i], w["wo"], g, None, None, r["a"][i], None, s)
            t.mm(r["a"][i].view(n, -1), w["wout"].t(), out=r["b"][i])
            Q.pnn_norm_fwd(r["sum"], r["b"][i], None, None, r["h"][i], w["wy"], r["h"][i + 1], r["y"][i + 1], s)
        return r["y"][-1]

    def forward(self, lengths=None, keep=None):
        """Logits of the loaded tokens; ``lengths``: int32, the tokens of each sequence that count; ``keep``: where the
        blocks' states after the last step go."""
        y = self._forward(self.whole, self.embed, self.tokens, None, keep, lengths)
        self.torch.mm(y, self.w.t(), out=self.logits)
        return self.logits

    def load(self, tokens, answers, advantage=None, old=None, ref=None):
        """tokens [batch][length]; per position: the token that was drawn from its logits (below 0: none), its advantage,
        and its log probability when it was drawn and of the reference (zeros where they are left out)."""
        self.tokens.copy_(tokens.view_as(self.tokens))
        self.answers.copy_(answers.reshape(-1))
        for dst, src in ((self.advantage, advantage), (self.old, old), (self.ref, ref)):
            if src is None:
                dst.zero_()
            else:
                dst.copy_(src.reshape(-1))

    def log_probabilities(self, lengths=None):
        """Of the loaded answers, [batch][length]; 0 where there is none."""
        self.forward(lengths)
        Q.pnn_policy_fwd_bwd(self.policy, self.logits, self.answers, self.advantage, None, self.ref, None, self.loss,
                             self.logp, None, self.stream())
        return self.logp.view(self.batch, self.length)

    def step(self, lengths=None):
        """Forward, loss and gradients: self.loss and self.logp [batch * length], self.dtable, and the other parameters'
        gradients as {name or (block, name): tensor}."""
        t, s, r = self.torch, self.stream(), self.whole
        self.forward(lengths)
        Q.pnn_policy_fwd_bwd(self.policy, self.logits, self.answers, self.advantage, self.old, self.ref, None, self.loss,
                             self.logp, self.logits, s)
        n, grads = self.n, {}
        grads["w"] = t.mm(self.logits.t(), r["y"][-1])
        t.mm(self.logits, self.w, out=r["dy"])
        new = lambda w: t.empty_like(w)
        dh = None                                            # the sum's gradient from later blocks
        for i in reversed(range(self.blocks)):
            w = self.layers[i]
            grads[i, "wy"], grads[i, "wo"] = new(w["wy"]), new(w["wo"])
            Q.pnn_norm_bwd(r["sum"], r["b"][i], None, None, r["h"][i], w["wy"], r["dy"], dh, r["db"], None, r["dh"], None,
                           grads[i, "wy"], False, self.ws, s)
            dh = r["dh"]
            grads[i, "wout"] = t.mm(r["db"].t(), r["a"][i].view(n, -1))
            t.mm(r["db"], w["wout"], out=r["da"].view(n, -1))
            q, k, v, g = self.split(r["p"][i])
            dq, dk, dv, dg = self.split(r["dp"])
            Q.pnn_norm_bwd(r["out"], r["o"][i], w["wo"], g, None, None, None, r["da"], r["do"], dg, None, grads[i, "wo"],
                           None, False, self.ws, s)
            Q.pnn_linattn_bwd(r["attn"], q, k, v, self.decay, lengths, None, r["do"], None, dq, dk, dv, None, self.ws, s)
            grads[i, "win"] = t.mm(r["dp"].view(n, -1).t(), r["y"][i])
            t.mm(r["dp"].view(n, -1), w["win"], out=r["dy"])
        grads["wy0"] = new(self.wy0)
        Q.pnn_norm_bwd(r["first"], r["h"][0], None, None, None, self.wy0, r["dy"], dh, r["db"], None, None, None,
                       grads["wy0"], False, self.ws, s)
        Q.pnn_embed_bwd(self.embed, r["db"], self.tokens, self.dtable, False, self.ws, s)
        return grads

    def update(self, grads, lr):
        """Plain gradient descent on every parameter."""
        self.table.add_(self.dtable.to(self.sdt), alpha=-lr)
        for name, g in grads.items():
            p = getattr(self, name) if isinstance(name, str) else self.layers[name[0]][name[1]]
            p.add_(g.to(p.dtype), alpha=-lr)

    def answer_step(self, noise):
        """One token of every sequence (self.token1): the next one, drawn with Gumbel noise [batch][vocab] (zeros: the
        most likely), in its place.  Nothing here looks at the host, so the step can be captured into a graph."""
        y = self._forward(self.one, self.embed1, self.token1, self.states, self.states)
        self.token1.copy_(self.draw(self.torch.mm(y, self.w.t()), noise))

    def draw(self, logits, noise):
        return (logits.float() / self.temperature + noise).argmax(1)

    def answer(self, tokens, noise, lengths=None):
        """Continues prompts [batch][length] (of ``lengths`` tokens, int32) by as many tokens as noise
        [steps][batch][vocab] has.  A prompt of no tokens has no logits: its first answer is drawn uniformly."""
        t = self.torch
        self.tokens.copy_(tokens.view_as(self.tokens))
        if lengths is not None:                              # what is behind a prompt's end is padding, whatever it holds
            self.tokens.masked_fill_(t.arange(self.length, device=self.dev) >= lengths[:, None], -1)
        logits = self.forward(lengths, keep=self.states).view(self.batch, self.length, -1)
        if lengths is None:
            last = logits[:, -1]
        else:
            last = logits[t.arange(self.batch, device=self.dev), lengths.long().clamp(1, self.length) - 1]
        out = t.empty(self.batch, len(noise), dtype=t.int64, device=self.dev)
        for i in range(len(noise)):
            if i == 0:
                self.token1.copy_(self.draw(last, noise[0]))
            else:
                self.answer_step(noise[i])
            out[:, i] = self.token1
        return out


def main():
    import torch
    vocab, batch, prompt, steps = 512, 64, 16, 48
    m = BlockModel(vocab, 256, 4, 64, 64, 2, batch, prompt + steps)
    asks = BlockModel(vocab, 256, 4, 64, 64, 2, batch, prompt)
    asks.table, asks.layers, asks.w, asks.wy0 = m.table, m.layers, m.w, m.wy0
    g = torch.Generator(device="cuda").manual_seed(1)
    prompts = torch.randint(0, vocab, (batch, prompt), generator=g, device="cuda")
    first = None
    for i in range(60):
        u = torch.rand(steps, batch, vocab, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)
        said = asks.answer(prompts, -torch.log(-torch.log(u)))
        tokens = torch.cat([prompts, said], 1)
        answers = torch.full_like(tokens, -1)
        answers[:, prompt - 1:-1] = said
        reward = (said % 2 == 0).float()
        m.load(tokens, answers)
        old = m.log_probabilities().clone()
        first = first if first is not None else old
        later = reward.flip(1).cumsum(1).flip(1) / torch.arange(steps, 0, -1, device="cuda")
        advantage = torch.zeros(batch, prompt + steps, device="cuda")
        advantage[:, prompt - 1:-1] = reward - reward.mean() + 0.1 * (later - later.mean())
        m.load(tokens, answers, advantage, old, old)
        for _ in range(2):
            m.update(m.step(), 4.0)
        if i % 10 == 0 or i == 59:
            print(f"step {i:3d}  even {reward.mean().item():.3f}  loss {m.loss.mean().item():.4f}", flush=True)
    print("answer", said[0, :8].tolist(), flush=True)


if __name__ == "__main__":
    main()
