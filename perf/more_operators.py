"""Performance cases of a sequence model's block and of the loss that trains it by its own answers.

Tokens' rows go through norms, through linear attention with a decay for each head, through a gate, and the policy's
logits are trained by a clipped policy loss.  Kinds (``kind``):

* ``lin_fwd``     o_t = scale q_t S_t with S_t = lambda_h S_{t-1} + k_t v_t^T: a prompt, or a single token with its state
* ``lin_train``   the same and its backward: gradients of the queries, keys, values and the first state
* ``norm_fwd``    h = res + alpha w1 norm(x) silu(gate), y = w2 norm(h), each part optional
* ``norm_train``  the same and its backward: gradients of every input and of both weights
* ``policy``      the clipped policy loss with a KL term of logits, log probabilities and the logits' gradient

``own = False`` computes them from elementary torch operations in 32 bits, ``own = True`` through the library.
``exact`` evaluates the definitions in 64 bits, the attention step by step.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------

def _lin(kind, batch, length, heads, kv, dk, dv, dtype="bf16", packed=False, ragged=False, state=True):
    # packed: queries, keys and values are parts of one projection's output, and so are their gradients
    return {"kind": kind, "batch": batch, "length": length, "heads": heads, "kv": kv, "dk": dk, "dv": dv,
            "dtype": dtype, "packed": packed, "ragged": ragged, "state": state}


def _norm(kind, rows, heads, width, dtype="bf16", post=True, gate=False, res=True, pre=True):
    return {"kind": kind, "rows": rows, "heads": heads, "width": width, "dtype": dtype, "post": post, "gate": gate,
            "res": res, "pre": pre}


def _policy(rows, classes, dtype="bf16", tau=1.0, kl=0.04, masked=False, old=True):
    return {"kind": "policy", "rows": rows, "classes": classes, "dtype": dtype, "tau": tau, "kl": kl, "masked": masked,
            "old": old}


def listed():
    def named(name, c):
        return {"name": name, **c}
    return [
        # answering: one new token of 64 sequences, their states read and written
        named("lin_token", _lin("lin_fwd", 64, 1, 16, 16, 128, 128)),
        # one long prompt, with the state it leaves
        named("lin_prompt", _lin("lin_fwd", 1, 32768, 16, 16, 128, 128, packed=True)),
        # a training batch of 8 sequences of 2048 tokens, from one projection
        named("lin_batch", _lin("lin_train", 8, 2048, 16, 16, 128, 128, packed=True, state=False)),
        # keys and values shared by four heads, sequences of different lengths that carry states
        named("lin_shared", _lin("lin_train", 4, 1024, 16, 4, 64, 128, ragged=True)),
        # odd sizes in fp32, sequences of different lengths (one of them empty)
        named("lin_odd", _lin("lin_train", 5, 777, 6, 2, 40, 72, "f32", ragged=True)),
        # answering: the residual sum and the next block's norm of 32 tokens (launch latency)
        named("norm_token", _norm("norm_fwd", 32, 1, 2048, post=False)),
        # a training batch: norm of a block's output, residual sum, norm before the next block
        named("norm_block", _norm("norm_train", 16384, 1, 2048)),
        # the norm of every head's output with its gate
        named("norm_heads", _norm("norm_train", 16384, 16, 128, gate=True, res=False, pre=False)),
        # odd sizes in fp32, every part at once
        named("norm_odd", _norm("norm_train", 1237, 1, 515, "f32", gate=True)),
        # the class count of the ImageNet-shaped head, a batch of 128
        named("policy_1000", _policy(128, 1000, "f32")),
        # a vocabulary: the largest
        named("policy_vocab", _policy(4096, 65536)),
        # an odd vocabulary, a sharper policy, prompts' tokens masked
        named("policy_odd", _policy(777, 32771, tau=0.7, masked=True)),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["lin_fwd", "lin_fwd", "lin_train", "lin_train", "norm_fwd", "norm_train", "norm_train",
                       "policy", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = SIZES[dtype]
    if kind in ("lin_fwd", "lin_train"):
        dk, dv = (rng.choice([_logint(rng, 8, 256), 64, 128]) for _ in range(2))
        kv = _logint(rng, 1, 16)
        heads = kv * rng.choice([1, 1, 2, 4])
        most = (1 << 25) // (heads * max(dk, dv)) * 2 // es
        length = rng.choice([1, _logint(rng, 1, min(16384, most)), _logint(rng, 64, min(16384, most))])
        batch = _logint(rng, 1, max(1, min(64, most // length, (1 << 24) // (heads * dk * dv))))
        return _lin(kind, batch, length, heads, kv, dk, dv, dtype, rng.random() < 0.5, rng.random() < 0.5,
                    rng.random() < 0.6)
    if kind in ("norm_fwd", "norm_train"):
        width = _logint(rng, 8, 8192)
        heads = rng.choice([1, 1, 1, _logint(rng, 2, 32)]) if width <= 512 else 1
        rows = _logint(rng, 1, (1 << 26) // (width * heads * es))
        res, gate = rng.random() < 0.6, rng.random() < 0.4
        pre = rng.random() < 0.6
        return _norm(kind, rows, heads, width, dtype, rng.random() < 0.6 or not pre, gate, res, pre)
    classes = _logint(rng, 10, 131072)
    rows = _logint(rng, 1, min(8192, (1 << 28) * 19 // (10 * classes * es)))
    return _policy(rows, classes, dtype, rng.choice([0.7, 1.0, 1.0, 1.5]), rng.choice([0.0, 0.04, 0.2]),
                   rng.random() < 0.5, rng.random() < 0.8)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _parts(c):
    """Queries, keys and values [batch][length][heads][width]: parts of one projection's rows, or apart."""
    B, T, dt = c["batch"], c["length"], DTYPES[c["dtype"]]
    size = [(c["heads"], c["dk"]), (c["kv"], c["dk"]), (c["kv"], c["dv"])]
    if not c["packed"]:
        return [torch.empty(B, T, h, w, device=DEV, dtype=dt) for h, w in size]
    rows = torch.empty(B, T, sum(h * w for h, w in size), device=DEV, dtype=dt)
    return [p.unflatten(2, s) for p, s in zip(rows.split([h * w for h, w in size], 2), size)]


def _prepare_lin(c, g):
    B, T, H, dk, dv, dt = c["batch"], c["length"], c["heads"], c["dk"], c["dv"], DTYPES[c["dtype"]]
    s = {"case": c, "scale": dk ** -0.5}
    s["q"], s["k"], s["v"] = _parts(c)
    for n in "qkv":
        s[n].copy_(_randn(g, *s[n].shape))
    # heads that keep a token for about 8 to 1024 steps
    s["decay"] = -torch.exp2(-3 - 7 * (torch.arange(H, device=DEV) + torch.rand(H, generator=g, device=DEV)) / H)
    s["lengths"] = None
    if c["ragged"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        if B > 1:
            s["lengths"][-1] = 0
    s["s0"] = _randn(g, B, H, dk, dv) if c["state"] else None
    s["sT"] = torch.empty(B, H, dk, dv, device=DEV) if c["state"] else None
    s["o"] = torch.empty(B, T, H, dv, device=DEV, dtype=dt)
    train = c["kind"] == "lin_train"
    if train:
        s["do"] = (_randn(g, B, T, H, dv) * 1e-2).to(dt)
        s["dsT"] = _randn(g, B, H, dk, dv) * 1e-2 if c["state"] else None
        s["dq"], s["dk"], s["dv"] = _parts(c)
        s["ds0"] = torch.empty(B, H, dk, dv, device=DEV) if c["state"] else None
    if own:
        from paper_2103_08802_amd import seq
        s["desc"] = seq.linattn_desc(s["q"], s["k"], s["v"], s["o"],
                                     *([s["do"], s["dq"], s["dk"], s["dv"]] if train else []), scale=s["scale"])
        fwd, bwd = seq.pnn_linattn_sizes(s["desc"])
        s["ws"] = torch.empty(max(fwd, bwd if train else 0, 256), device=DEV, dtype=torch.uint8)
    return s


def _prepare_norm(c, g):
    dt, shape = DTYPES[c["dtype"]], (c["rows"], c["heads"], c["width"])
    s = {"case": c, "alpha": 0.5 if c["res"] else 1.0}
    some = lambda on: _randn(g, *shape).to(dt) if on else None
    s["x"], s["gate"], s["res"] = some(True), some(c["gate"]), some(c["res"])
    weight = lambda on: 1 + 0.2 * _randn(g, c["width"]) if on else None
    s["w1"], s["w2"] = weight(c["post"]), weight(c["pre"])
    empty = lambda on: torch.empty(shape, device=DEV, dtype=dt) if on else None
    train = c["kind"] == "norm_train"
    # the sum is kept where another block adds to it or the backward needs it
    s["h"], s["y"] = empty(c["res"] or not c["pre"] or train), empty(c["pre"])
    if train:
        s["dy"] = (_randn(g, *shape) * 1e-2).to(dt) if c["pre"] else None
        s["dh"] = (_randn(g, *shape) * 1e-2).to(dt) if c["res"] or not c["pre"] else None
        s["dx"], s["dgate"], s["dres"] = empty(True), empty(c["gate"]), empty(c["res"])
        s["dw1"], s["dw2"] = (None if w is None else torch.empty(c["width"], device=DEV) for w in (s["w1"], s["w2"]))
    if own:
        from paper_2103_08802_amd import seq
        more = {n: s[n] for n in ("dy", "dh", "dx", "dgate", "dres")} if train else {}
        s["desc"] = seq.norm_desc(s["x"], gate=s["gate"], res=s["res"], h=s["h"], y=s["y"], **more, post=c["post"],
                                  pre=c["pre"], eps=EPS, alpha=s["alpha"], kept=train)
        if train:
            s["ws"] = torch.empty(max(seq.pnn_norm_workspace_size(s["desc"]), 256), device=DEV, dtype=torch.uint8)
    return s


LOW, HIGH = 0.2, 0.28


def _prepare_policy(c, g):
    n, v, dt = c["rows"], c["classes"], DTYPES[c["dtype"]]
    # a policy that is sure of some tokens and unsure of others; the answers are drawn from it
    z = torch.empty(n, v, device=DEV, dtype=dt)
    z.copy_(_randn(g, n, v))
    z *= 1 + 2 * torch.rand(n, 1, generator=g, device=DEV).to(dt)
    s = {"case": c, "logits": z, "scale": 1.0 / n}
    part = max(1, (1 << 26) // v)
    token, lp = [], []
    for r in range(0, n, part):
        t = z[r:r + part].double() / c["tau"]
        noise = -torch.log(torch.empty(t.shape, device=DEV).exponential_(generator=g))
        a = (t + noise).argmax(1, keepdim=True)
        token.append(a[:, 0])
        lp.append((t.gather(1, a) - torch.logsumexp(t, 1, keepdim=True))[:, 0])
    lp = torch.cat(lp)
    s["tokens"] = torch.cat(token).to(torch.int32)
    if c["masked"]:
        s["tokens"][torch.rand(n, generator=g, device=DEV) < 0.3] = -1
    s["advantage"] = _randn(g, n)
    # a few updates behind; the ratio is kept off the borders, where the loss has a step in its gradient
    off = 0.25 * _randn(g, n)
    for border in (math.log(1 - LOW), math.log(1 + HIGH)):
        off = torch.where((off - border).abs() < 1e-3, torch.full_like(off, 0.01), off)
    s["old"] = (lp - off).float() if c["old"] else None
    s["ref"] = (lp + 0.3 * _randn(g, n)).float() if c["kl"] != 0 else None
    s["weight"] = torch.rand(n, generator=g, device=DEV) + 0.5 if c["masked"] else None
    s["loss"], s["logp"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    s["dlogits"] = torch.empty(n, v, device=DEV, dtype=dt)
    if own:
        from paper_2103_08802_amd import seq
        s["desc"] = seq.policy_desc(z, s["dlogits"], c["tau"], LOW, HIGH, c["kl"], s["scale"])
    return s


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"].startswith("lin"):
        return _prepare_lin(case, g)
    if case["kind"].startswith("norm"):
        return _prepare_norm(case, g)
    return _prepare_policy(case, g)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

CHUNK = 128


def _plain_linear(q, k, v, decay):
    """o_t = sum over s <= t of lambda^(t - s) (q_t k_s) v_s, [batch][heads][length][width], in chunks."""
    B, H, T, _ = q.shape
    C = min(CHUNK, T)
    N = -(-T // C)
    cut = lambda t: torch.nn.functional.pad(t, (0, 0, 0, N * C - T)).unflatten(2, (N, C))
    q, k, v = cut(q), cut(k), cut(v)
    i = torch.arange(C, device=DEV, dtype=torch.float32)
    d = decay[:, None, None]
    apart = i[:, None] - i
    D = torch.where(apart >= 0, torch.exp(d * apart.clamp(min=0)), torch.zeros((), device=DEV))
    o = torch.matmul(torch.matmul(q, k.transpose(3, 4)) * D[:, None], v)
    if N > 1:
        late = torch.exp(d * (C - 1 - i)[:, None])[:, None]
        U = torch.matmul((k * late).transpose(3, 4), v)
        n = torch.arange(N, device=DEV, dtype=torch.float32)
        far = n[:, None] - 1 - n
        M = torch.where(far >= 0, torch.exp(d * C * far.clamp(min=0)), torch.zeros((), device=DEV))
        S = torch.matmul(M, U.flatten(3)).unflatten(3, U.shape[3:])
        o += torch.matmul(q * torch.exp(d * (i + 1)[:, None])[:, None], S)
    return o.flatten(2, 3)[:, :, :T]


def _plain_lin(s):
    c = s["case"]
    T, H, dt, scale = c["length"], c["heads"], s["q"].dtype, s["scale"]
    t = torch.arange(T, device=DEV)
    B = c["batch"]
    n = s["lengths"].long().clamp(0, T) if s["lengths"] is not None else torch.full((B,), T, device=DEV)
    live = (t < n[:, None])[:, None, :, None]
    zero = torch.zeros((), device=DEV)
    heads = lambda x: torch.where(live, x.float().transpose(1, 2).repeat_interleave(H // x.shape[2], 1), zero)
    rows = lambda x, like: x.transpose(1, 2).unflatten(2, (like.shape[2], -1)).sum(3).to(dt)
    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    d = s["decay"]
    since = torch.where(live, torch.exp(d[:, None, None] * (t[:, None] + 1)), zero)             # lambda^(t + 1)
    until = torch.where(live, torch.exp(d[:, None, None] * (n[:, None, None, None] - 1 - t[:, None])), zero)
    o = _plain_linear(q, k, v, d)
    if c["state"]:
        o = o + torch.matmul(q * since, s["s0"])
    out = [rows(o * scale, s["q"])]
    if c["state"]:
        gone = torch.exp(d[:, None, None] * n[:, None, None, None])                             # lambda^n
        out.append(gone * s["s0"] + torch.matmul((k * until).transpose(2, 3), v))
    if c["kind"] == "lin_fwd":
        return out
    do = heads(s["do"]) * scale
    dq = _plain_linear(do, v, k, d)
    back = lambda x: x.flip(2)
    dk = back(_plain_linear(back(v), back(do), back(q), d))
    dv = back(_plain_linear(back(k), back(q), back(do), d))
    if c["state"]:
        dq = dq + torch.matmul(do * since, s["s0"].transpose(2, 3))
        dk = dk + torch.matmul(v * until, s["dsT"].transpose(2, 3))
        dv = dv + torch.matmul(k * until, s["dsT"])
    out += [rows(dq, s["q"]), rows(dk, s["k"]), rows(dv, s["v"])]
    if c["state"]:
        out.append(gone * s["dsT"] + torch.matmul((q * since).transpose(2, 3), do))
    return out


def _plain_norm_of(u):
    return u / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)


def _plain_norm_back(u, dn):
    r = 1 / torch.sqrt((u * u).mean(-1, keepdim=True) + EPS)
    n = u * r
    return r * (dn - n * (dn * n).mean(-1, keepdim=True))


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    n = _plain_norm_of(x) if c["post"] else x
    a = n * s["w1"] if c["post"] else n
    if c["gate"]:
        gate = s["gate"].float()
        sig = 1 / (1 + torch.exp(-gate))
        swish = gate * sig
    h = s["alpha"] * (a * swish if c["gate"] else a)
    if c["res"]:
        h = h + s["res"].float()
    out = [h.to(dt)] if s["h"] is not None else []
    if c["pre"]:
        out.append((_plain_norm_of(h) * s["w2"]).to(dt))
    if c["kind"] == "norm_fwd":
        return out
    dh = torch.zeros_like(h) if s["dh"] is None else s["dh"].float()
    dw = []
    if c["pre"]:
        dy = s["dy"].float()
        dh = dh + _plain_norm_back(h, dy * s["w2"])
        dw.append((dy * _plain_norm_of(h)).sum((0, 1)))
    g = s["alpha"] * dh
    grads = []
    if c["gate"]:
        grads.append((g * a * (sig + swish * (1 - sig))).to(dt))
        g = g * swish
    if c["post"]:
        dw.append((g * n).sum((0, 1)))
        g = _plain_norm_back(x, g * s["w1"])
    return out + [g.to(dt)] + grads + ([dh.to(dt)] if c["res"] else []) + dw


def _plain_policy(s):
    c = s["case"]
    z = s["logits"].float()
    t = z if c["tau"] == 1.0 else z / c["tau"]
    held = s["tokens"] >= 0
    a = s["tokens"].long().clamp(min=0)[:, None]
    m = t.amax(1, keepdim=True)
    p = torch.exp(t - m)
    total = p.sum(1, keepdim=True)
    # log probabilities by their difference to the old ones: 64 bits next to the clip's borders
    lp = ((t.gather(1, a) - m).double() - torch.log(total.double()))[:, 0]
    A = s["advantage"].double()
    r = torch.exp(lp - s["old"].double()) if c["old"] else torch.ones_like(lp)
    plain, cut = r * A, r.clamp(1 - LOW, 1 + HIGH) * A
    loss = -torch.minimum(plain, cut)
    slope = torch.where(plain <= cut, -plain, torch.zeros_like(plain))
    if c["kl"] != 0:
        apart = s["ref"].double() - lp
        loss = loss + c["kl"] * (torch.expm1(apart) - apart)
        slope = slope - c["kl"] * torch.expm1(apart)
    none = torch.zeros((), device=DEV, dtype=torch.float64)
    slope = torch.where(held, slope, none) * (s["scale"] / c["tau"])
    if s["weight"] is not None:
        slope = slope * s["weight"].double()
    slope = slope.float()[:, None]
    p *= -slope / total
    p.scatter_add_(1, a, slope)
    return [torch.where(held, loss, none).float(), torch.where(held, lp, none).float(), p.to(s["logits"].dtype)]


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if not own:
        return _plain_policy(s) if kind == "policy" else _plain_lin(s) if kind.startswith("lin") else _plain_norm(s)
    from paper_2103_08802_amd import seq
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "policy":
        seq.pnn_policy_fwd_bwd(s["desc"], s["logits"], s["tokens"], s["advantage"], s["old"], s["ref"], s["weight"],
                               s["loss"], s["logp"], s["dlogits"], stream)
        return [s["loss"], s["logp"], s["dlogits"]]
    if kind.startswith("lin"):
        seq.pnn_linattn_fwd(s["desc"], s["q"], s["k"], s["v"], s["decay"], s["lengths"], s["s0"], s["o"], s["sT"],
                            s["ws"], stream)
        out = [s["o"]] + ([s["sT"]] if c["state"] else [])
        if kind == "lin_train":
            seq.pnn_linattn_bwd(s["desc"], s["q"], s["k"], s["v"], s["decay"], s["lengths"], s["s0"], s["do"], s["dsT"],
                                s["dq"], s["dk"], s["dv"], s["ds0"], s["ws"], stream)
            out += [s["dq"], s["dk"], s["dv"]] + ([s["ds0"]] if c["state"] else [])
        return out
    seq.pnn_norm_fwd(s["desc"], s["x"], s["w1"], s["gate"], s["res"], s["w2"], s["h"], s["y"], stream)
    out = [s["h"], s["y"]]
    if kind == "norm_train":
        seq.pnn_norm_bwd(s["desc"], s["x"], s["w1"], s["gate"], s["h"], s["w2"], s["dy"], s["dh"], s["dx"], s["dgate"],
                         s["dres"], s["dw1"], s["dw2"], False, s["ws"], stream)
        out += [s["dx"], s["dgate"], s["dres"], s["dw2"], s["dw1"]]
    return [t for t in out if t is not None]


# ------------------------------------------------------------------------------------------------
# the least work, and the definitions in 64 bits
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    es = SIZES[c["dtype"]]
    if c["kind"].startswith("lin"):
        H, kv, dk, dv = c["heads"], c["kv"], c["dk"], c["dv"]
        tokens = c["batch"] * c["length"]
        part = c["batch"] * H * dk * dv * 4 if c["state"] else 0
        one = tokens * (H * (dk + dv) + kv * (dk + dv)) * es
        if c["kind"] == "lin_fwd":
            return {"bytes": one + 2 * part, "flops": 4 * tokens * H * dk * dv}
        # the backward's inputs are those the forward read
        return {"bytes": 2 * one + 4 * part, "flops": 14 * tokens * H * dk * dv}
    if c["kind"].startswith("norm"):
        one = c["rows"] * c["heads"] * c["width"]
        train = c["kind"] == "norm_train"
        read = 1 + c["gate"] + c["res"]
        written = (c["res"] or not c["pre"] or train) + c["pre"]
        if train:
            read += c["pre"] + (c["res"] or not c["pre"])
            written += 1 + c["gate"] + c["res"]
        return {"bytes": (read + written) * one * es, "flops": one * (30 if train else 10)}
    rows = c["rows"] * c["classes"]
    return {"bytes": 2 * rows * es + 28 * c["rows"], "flops": 7 * rows}


def _exact_lin(s):
    c = s["case"]
    B, T, H = c["batch"], c["length"], c["heads"]
    wide = lambda t: t.to(torch.float64).permute(1, 0, 2, 3).repeat_interleave(H // t.shape[2], 2)
    q, k, v = wide(s["q"]), wide(s["k"]), wide(s["v"])
    lam = torch.exp(s["decay"].to(torch.float64))[:, None, None]
    n = torch.full((B,), T, device=DEV) if s["lengths"] is None else s["lengths"].long()
    live = torch.arange(T, device=DEV)[:, None] < n
    masked = bool((~live).any())
    S = (torch.zeros(B, H, c["dk"], c["dv"], device=DEV, dtype=torch.float64) if s["s0"] is None
         else s["s0"].to(torch.float64))
    train = c["kind"] == "lin_train"
    if train:
        do = wide(s["do"]) * s["scale"]
    o, dq, dk, dv = [], [], [], []
    for t in range(T):
        m = live[t][:, None, None, None]
        new = torch.addcmul(lam * S, k[t][..., None], v[t][:, :, None])
        S = torch.where(m, new, S) if masked else new
        o.append(torch.matmul(q[t][:, :, None], S)[:, :, 0] * s["scale"])
        if train:
            dq.append(torch.matmul(S, do[t][..., None])[..., 0])
    fold = lambda x, heads: (torch.stack(x) * live[..., None, None]).transpose(0, 1).unflatten(2, (heads, -1)).sum(3)
    out = [fold(o, H)] + ([S] if c["state"] else [])
    if not train:
        return out
    Z = torch.zeros_like(S) if s["dsT"] is None else s["dsT"].to(torch.float64)
    for t in range(T - 1, -1, -1):
        m = live[t][:, None, None, None]
        at = torch.addcmul(Z, q[t][..., None], do[t][:, :, None])
        dk.append(torch.matmul(at, v[t][..., None])[..., 0])
        dv.append(torch.matmul(k[t][:, :, None], at)[:, :, 0])
        Z = torch.where(m, lam * at, Z)
    out += [fold(dq, H), fold(dk[::-1], c["kv"]), fold(dv[::-1], c["kv"])]
    return out + ([Z] if c["state"] else [])


def _exact_norm(s):
    c = s["case"]
    wide = lambda t: None if t is None else t.to(torch.float64).requires_grad_()
    x, gate, res, w1, w2 = (wide(s[n]) for n in ("x", "gate", "res", "w1", "w2"))
    rms = lambda u: u * torch.rsqrt(u.pow(2).mean(-1, keepdim=True) + EPS)
    a = rms(x) * w1 if c["post"] else x
    if gate is not None:
        a = a * (gate * torch.sigmoid(gate))
    h = s["alpha"] * a + (0 if res is None else res)
    y = rms(h) * w2 if c["pre"] else None
    out = [h] if s["h"] is not None else []
    out += [y] if c["pre"] else []
    if c["kind"] == "norm_train":
        ends, seeds = [], []
        for t, d in ((h, s["dh"]), (y, s["dy"])):
            if t is not None and d is not None:
                ends.append(t)
                seeds.append(d.to(torch.float64))
        leaves = [t for t in (x, gate, res, w2, w1) if t is not None]
        out += list(torch.autograd.grad(ends, leaves, seeds))
    return [t.detach() for t in out]


def _exact_policy(s):
    c = s["case"]
    loss, logp, grad = [], [], []
    part = max(1, (1 << 27) // c["classes"])
    for r in range(0, c["rows"], part):
        at = slice(r, r + part)
        lg = torch.log_softmax(s["logits"][at].to(torch.float64) / c["tau"], 1)
        a = s["tokens"][at].long()
        held = a >= 0
        pick = torch.arange(len(a), device=DEV), a.clamp(min=0)
        lp = lg[pick].requires_grad_()
        A = s["advantage"][at].to(torch.float64)
        ratio = torch.exp(lp - (s["old"][at].to(torch.float64) if c["old"] else lp.detach()))
        each = -torch.min(ratio * A, ratio.clamp(1 - LOW, 1 + HIGH) * A)
        if c["kl"] != 0:
            x = s["ref"][at].to(torch.float64) - lp
            each = each + c["kl"] * (torch.exp(x) - x - 1)
        each = torch.where(held, each, 0.0)
        slope, = torch.autograd.grad(each.sum(), lp)
        slope = slope * s["scale"] / c["tau"] * (1 if s["weight"] is None else s["weight"][at].to(torch.float64))
        d = torch.exp(lg) * -slope[:, None]
        d[pick] += slope
        loss.append(each.detach())
        logp.append(torch.where(held, lp.detach(), 0.0))
        grad.append(d.to(torch.float32) if d.numel() * 8 > (1 << 28) else d)
    if len(grad) > 1:
        grad = [t.to(torch.float32) for t in grad]
    return [torch.cat(loss), torch.cat(logp), torch.cat(grad)]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "policy":
        return _exact_policy(s)
    return _exact_lin(s) if case["kind"].startswith("lin") else _exact_norm(s)
