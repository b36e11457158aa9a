"""Performance cases of the sequence operators: token embedding, gated linear recurrence, distillation loss.

A sequence model takes token ids through an embedding, runs a recurrence along the sequence and is trained towards a
teacher's largest logits.  Kinds (``kind``):

* ``embed_fwd``   rows of a table, scaled, for a list of tokens
* ``embed_bwd``   the table's gradient (fp32) from the rows' gradients, over one or two micro-batches: the first
                  overwrites the gradient, the second adds to it
* ``scan_fwd``    h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(gate): a prompt, or a single token with its state
* ``scan_train``  the same and its backward: gradients of the inputs, the gates and the first state
* ``distill``     loss and logit gradients from a teacher's top logits, with or without labels

``own = False`` computes them from elementary torch operations in 32 bits, ``own = True`` through the library.
``exact`` evaluates the definitions in 64 bits, step by step.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------

def _embed(kind, n, width, vocab, dtype="bf16", token="i64", micro=1):
    return {"kind": kind, "n": n, "width": width, "vocab": vocab, "dtype": dtype, "token": token, "micro": micro}


def _scan(kind, batch, length, channels, dtype="bf16", layout="dense", ragged=False, state=True):
    # layout "halves": inputs and gates are the two halves of one projection's output, and so are their gradients
    return {"kind": kind, "batch": batch, "length": length, "channels": channels, "dtype": dtype, "layout": layout,
            "ragged": ragged, "state": state}


def _distill(rows, classes, top, dtype="bf16", tau=2.0, alpha=0.5, labels=True, ragged=False):
    return {"kind": "distill", "rows": rows, "classes": classes, "top": top, "dtype": dtype, "tau": tau,
            "alpha": alpha, "labels": labels, "ragged": ragged}


def listed():
    def named(name, c):
        return {"name": name, **c}
    return [
        # answering: one new token for each of 32 sequences (launch latency)
        named("embed_token", _embed("embed_fwd", 32, 1024, 32768)),
        # a training batch of 8 sequences of 2048 tokens
        named("embed_batch", _embed("embed_fwd", 16384, 2048, 65536)),
        # its gradient, into a table of which the batch touches a part
        named("embed_grad", _embed("embed_bwd", 16384, 2048, 65536)),
        # two large micro-batches over a small vocabulary: long runs of equal tokens
        named("embed_grad_micro", _embed("embed_bwd", 65536, 1024, 8192, micro=2)),
        # odd sizes in fp32, 32-bit tokens
        named("embed_grad_odd", _embed("embed_bwd", 1237, 515, 10007, "f32", "i32")),
        # answering: one step of 64 sequences with their states
        named("scan_token", _scan("scan_fwd", 64, 1, 2048)),
        # one long prompt
        named("scan_prompt", _scan("scan_fwd", 1, 65536, 1024)),
        # a training batch, inputs and gates from one projection
        named("scan_batch", _scan("scan_train", 8, 2048, 2048, layout="halves", state=False)),
        # odd sizes in fp32, sequences of different lengths (one of them empty)
        named("scan_ragged", _scan("scan_train", 5, 777, 333, "f32", ragged=True)),
        # the class count of the ImageNet-shaped head, a batch of 128, no tempering
        named("distill_1000", _distill(128, 1000, 10, "f32", tau=1.0)),
        # a vocabulary: the largest
        named("distill_vocab", _distill(4096, 65536, 64)),
        # an odd vocabulary, rows with few or no teacher entries and rows without a label
        named("distill_odd", _distill(777, 32771, 20, ragged=True)),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_bwd", "scan_fwd", "scan_train", "scan_train", "distill", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = SIZES[dtype]
    if kind in ("embed_fwd", "embed_bwd"):
        width = _logint(rng, 8, 4096)
        n = _logint(rng, 1, min(131072, (1 << 28) // (width * es)))
        vocab = _logint(rng, 64, min(262144, (1 << 28) // (width * 4)))
        return _embed(kind, n, width, vocab, dtype, rng.choice(["i32", "i64"]),
                      rng.choice([1, 2]) if kind == "embed_bwd" else 1)
    if kind in ("scan_fwd", "scan_train"):
        channels = _logint(rng, 8, 4096)
        length = _logint(rng, 1, 65536)
        batch = _logint(rng, 1, max(1, min(64, (1 << 27) // (channels * length * es))))
        length = min(length, max(1, (1 << 27) // (channels * batch * es)))
        return _scan(kind, batch, length, channels, dtype, rng.choice(["dense", "halves"]),
                     rng.random() < 0.5, rng.random() < 0.5)
    classes = _logint(rng, 10, 131072)
    rows = _logint(rng, 1, min(8192, (1 << 28) * 19 // (10 * classes * es)))
    return _distill(rows, classes, _logint(rng, 1, min(128, classes)), dtype, rng.choice([1.0, 2.0, 4.0]),
                    rng.choice([0.5, 0.9, 1.0]), rng.random() < 0.6, rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tokens(g, n, vocab, dtype):
    """Token ids as often as words are: id v with probability log((v + 2) / (v + 1)) / log(vocab + 1); one in 33 is
    padding (-1)."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    pad = torch.randint(0, 33, (n,), generator=g, device=DEV) == 0
    return torch.where(pad, torch.full_like(t, -1), t).to(torch.int64 if dtype == "i64" else torch.int32)


def _distinct(n, vocab):
    """Expected number of different tokens among n."""
    v = torch.arange(vocab, dtype=torch.float64)
    p = 32 / 33 * torch.log((v + 2) / (v + 1)) / math.log(vocab + 1)
    return float((1 - torch.exp(n * torch.log1p(-p))).sum())


def _prepare_embed(c, g):
    dt, w = DTYPES[c["dtype"]], c["width"]
    s = {"case": c, "scale": math.sqrt(w)}
    s["tokens"] = [_tokens(g, c["n"], c["vocab"], c["token"]) for _ in range(c["micro"])]
    if c["kind"] == "embed_fwd":
        s["table"] = (torch.randn(c["vocab"], w, generator=g, device=DEV) * w ** -0.5).to(dt)
        s["out"] = torch.empty(c["n"], w, device=DEV, dtype=dt)
    else:
        s["dout"] = [(torch.randn(c["n"], w, generator=g, device=DEV) * 1e-2).to(dt) for _ in range(c["micro"])]
        s["dtable"] = torch.empty(c["vocab"], w, device=DEV, dtype=torch.float32)
    if own:
        from paper_2103_08802_amd import seq
        if c["kind"] == "embed_fwd":
            s["desc"] = seq.embed_desc(s["table"], s["tokens"][0], s["out"], s["scale"])
        else:
            s["desc"] = seq.embed_desc(s["dtable"], s["tokens"][0], s["dout"][0], s["scale"])
            s["ws"] = torch.empty(seq.pnn_embed_workspace_size(s["desc"]), device=DEV, dtype=torch.uint8)
    return s


def _pair(c, fill):
    """Two [batch][length][channels] tensors, dense or as the halves of one."""
    shape = (c["batch"], c["length"], c["channels"])
    dt = DTYPES[c["dtype"]]
    if c["layout"] == "halves":
        both = torch.empty(shape[0], shape[1], 2 * shape[2], device=DEV, dtype=dt)
        a, b = both[..., :shape[2]], both[..., shape[2]:]
    else:
        a, b = torch.empty(shape, device=DEV, dtype=dt), torch.empty(shape, device=DEV, dtype=dt)
    if fill is not None:
        a.copy_(fill[0])
        b.copy_(fill[1])
    return a, b


def _prepare_scan(c, g):
    dt = DTYPES[c["dtype"]]
    shape = (c["batch"], c["length"], c["channels"])
    # gates that keep a state for one step to a few hundred, by channel
    gate = torch.randn(shape, generator=g, device=DEV)
    gate += torch.rand(c["channels"], generator=g, device=DEV) * 8 - 2
    s = {"case": c}
    s["x"], s["gate"] = _pair(c, (torch.randn(shape, generator=g, device=DEV), gate))
    s["lengths"] = None
    if c["ragged"]:
        s["lengths"] = torch.randint(0, c["length"] + 1, (c["batch"],), generator=g, device=DEV, dtype=torch.int32)
        s["lengths"][-1] = 0
    s["h0"] = torch.randn(c["batch"], c["channels"], generator=g, device=DEV) * 0.5 if c["state"] else None
    s["h"] = torch.empty(shape, device=DEV, dtype=dt)
    s["hT"] = torch.empty(c["batch"], c["channels"], device=DEV) if c["state"] else None
    train = c["kind"] == "scan_train"
    if train:
        s["dh"] = (torch.randn(shape, generator=g, device=DEV) * 1e-2).to(dt)
        s["dhT"] = torch.randn(c["batch"], c["channels"], generator=g, device=DEV) * 1e-2 if c["state"] else None
        s["dx"], s["dgate"] = _pair(c, None)
        s["dh0"] = torch.empty(c["batch"], c["channels"], device=DEV) if c["state"] else None
    if own:
        from paper_2103_08802_amd import seq
        s["desc"] = seq.scan_desc(s["x"], s["gate"], s["h"], *([s["dh"], s["dx"], s["dgate"]] if train else []))
        states, ws = seq.pnn_scan_sizes(s["desc"])
        s["states"] = torch.empty(max(states // 4, 1), device=DEV) if train else None
        s["ws"] = torch.empty(max(ws, 256), device=DEV, dtype=torch.uint8)
    return s


def _prepare_distill(c, g):
    n, v, k = c["rows"], c["classes"], c["top"]
    step = torch.randint(1, max(v // k, 1) + 1, (n, 1), generator=g, device=DEV)
    first = torch.randint(0, v, (n, 1), generator=g, device=DEV)
    index = (first + step * torch.arange(k, device=DEV)) % v                 # k different classes
    teacher = 9 - torch.empty(n, k, device=DEV).exponential_(0.5, generator=g).cumsum(1) / math.sqrt(k)
    z = torch.randn(n, v, generator=g, device=DEV)
    z.scatter_add_(1, index, 0.8 * teacher.clamp(min=0))
    labels = index[:, 0].to(torch.int32)
    if c["ragged"]:
        held = torch.randint(0, k + 1, (n, 1), generator=g, device=DEV)      # entries of a row: none up to all
        index = torch.where(torch.arange(k, device=DEV) < held, index, torch.full_like(index, -1))
        labels = torch.where(torch.rand(n, generator=g, device=DEV) < 0.2, torch.full_like(labels, -1), labels)
    dt = DTYPES[c["dtype"]]
    s = {"case": c, "logits": z.to(dt), "index": index.to(torch.int32), "teacher": teacher.to(dt),
         "labels": labels if c["labels"] else None, "scale": 1.0 / n,
         "weight": torch.rand(n, generator=g, device=DEV) + 0.5 if c["ragged"] else None}
    s["loss"] = torch.empty(n, device=DEV)
    s["dlogits"] = torch.empty(n, v, device=DEV, dtype=dt)
    if own:
        from paper_2103_08802_amd import seq
        s["desc"] = seq.distill_desc(s["logits"], s["teacher"], s["dlogits"], c["tau"], c["alpha"], s["scale"])
    return s


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"].startswith("embed"):
        return _prepare_embed(case, g)
    if case["kind"].startswith("scan"):
        return _prepare_scan(case, g)
    return _prepare_distill(case, g)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _plain_embed_fwd(s):
    t = s["tokens"][0].long()
    rows = s["table"][t.clamp(min=0)].float() * s["scale"]
    return torch.where((t >= 0)[:, None], rows, torch.zeros_like(rows)).to(s["table"].dtype)


def _plain_embed_bwd(s):
    total = torch.zeros_like(s["dtable"])
    for t, dout in zip(s["tokens"], s["dout"]):
        t = t.long()
        rows = torch.where((t >= 0)[:, None], dout.float(), torch.zeros((), device=DEV))
        total.index_add_(0, t.clamp(min=0), rows * s["scale"])
    return total


def _plain_chain(a, b):
    """y_t = a_t y_{t-1} + b_t along dim 1 from y_{-1} = 0, by doubling."""
    d, length = 1, a.shape[1]
    while d < length:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _plain_scan(s):
    c = s["case"]
    dt = s["x"].dtype
    x, gate = s["x"].float(), s["gate"].float()
    f = 1 / (1 + torch.exp(-gate))
    keep = 1 / (1 + torch.exp(gate))                                         # 1 - f
    live = None
    zero = torch.zeros((), device=DEV)
    one = torch.ones((), device=DEV)
    b = keep * x
    if s["lengths"] is not None:
        live = (torch.arange(c["length"], device=DEV) < s["lengths"][:, None])[..., None]
        f, b = torch.where(live, f, one), torch.where(live, b, zero)
    first = s["h0"] if s["h0"] is not None else torch.zeros(c["batch"], c["channels"], device=DEV)
    h = _plain_chain(f, torch.cat([b[:, :1] + f[:, :1] * first[:, None], b[:, 1:]], 1))
    out = [(h if live is None else torch.where(live, h, zero)).to(dt)]
    if c["state"]:
        out.append(h[:, -1].clone())
    if c["kind"] == "scan_fwd":
        return out
    dh = s["dh"].float()
    if live is not None:
        dh = torch.where(live, dh, zero)
    last = dh[:, -1:] + s["dhT"][:, None] if c["state"] else dh[:, -1:]
    later = torch.cat([f[:, 1:], torch.zeros_like(f[:, :1])], 1)
    G = _plain_chain(later.flip(1), torch.cat([dh[:, :-1], last], 1).flip(1)).flip(1)
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    dx, dgate = G * keep, G * (before - x) * f * keep
    if live is not None:
        dx, dgate = torch.where(live, dx, zero), torch.where(live, dgate, zero)
    out += [dx.to(dt), dgate.to(dt)]
    if c["state"]:
        out.append(f[:, 0] * G[:, 0])
    return out


def _plain_softmax(z):
    """exp(z - max) / sum and the logarithm of sum exp(z)."""
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    return e / total, m + torch.log(total)


def _plain_distill(s):
    c = s["case"]
    tau, alpha = c["tau"], c["alpha"]
    z = s["logits"].float()
    held = s["index"] >= 0
    index = s["index"].long().clamp(min=0)
    t = torch.where(held, s["teacher"].float() / tau, torch.full((), -math.inf, device=DEV))
    some = held.any(1, keepdim=True)
    p, tl = _plain_softmax(torch.where(some, t, torch.zeros((), device=DEV)))
    zero = torch.zeros((), device=DEV)
    p = torch.where(held, p, zero)
    q, ql = _plain_softmax(z / tau)
    kl = torch.where(held, p * ((t - tl) - (z.gather(1, index) / tau - ql)), zero).sum(1)
    loss = alpha * tau * tau * kl
    d = torch.where(some, q, zero).scatter_add_(1, index, -p) * (alpha * tau)
    if s["labels"] is not None:
        known = s["labels"] >= 0
        y = s["labels"].long().clamp(min=0)[:, None]
        sm, sl = _plain_softmax(z)
        loss = loss + (1 - alpha) * torch.where(known, (sl - z.gather(1, y))[:, 0], zero)
        hard = sm.scatter_add_(1, y, torch.full_like(sl, -1.0))
        d += (1 - alpha) * torch.where(known[:, None], hard, zero)
    d *= s["scale"] if s["weight"] is None else (s["scale"] * s["weight"])[:, None]
    return [loss, d.to(s["logits"].dtype)]


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        if kind == "embed_fwd":
            return _plain_embed_fwd(s)
        if kind == "embed_bwd":
            return _plain_embed_bwd(s)
        return _plain_distill(s) if kind == "distill" else _plain_scan(s)
    from paper_2103_08802_amd import seq
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "embed_fwd":
        seq.pnn_embed_fwd(s["desc"], s["table"], s["tokens"][0], s["out"], stream)
        return s["out"]
    if kind == "embed_bwd":
        for i, (t, dout) in enumerate(zip(s["tokens"], s["dout"])):
            seq.pnn_embed_bwd(s["desc"], dout, t, s["dtable"], i > 0, s["ws"], stream)
        return s["dtable"]
    if kind == "distill":
        seq.pnn_distill_fwd_bwd(s["desc"], s["logits"], s["index"], s["teacher"], s["labels"], s["weight"], s["loss"],
                                s["dlogits"], stream)
        return [s["loss"], s["dlogits"]]
    seq.pnn_scan_fwd(s["desc"], s["x"], s["gate"], s["lengths"], s["h0"], s["h"], s["hT"], s["states"], s["ws"], stream)
    out = [s["h"]] + ([s["hT"]] if s["hT"] is not None else [])
    if kind == "scan_train":
        seq.pnn_scan_bwd(s["desc"], s["x"], s["gate"], s["lengths"], s["states"], s["dh"], s["dhT"], s["dx"],
                         s["dgate"], s["dh0"], s["ws"], stream)
        out += [s["dx"], s["dgate"]] + ([s["dh0"]] if s["dh0"] is not None else [])
    return out


# ------------------------------------------------------------------------------------------------
# the least work, and the definitions in 64 bits
# ------------------------------------------------------------------------------------------------

def work(case):
    c = case
    es = SIZES[c["dtype"]]
    if c["kind"].startswith("embed"):
        tb = 8 if c["token"] == "i64" else 4
        rows = c["n"] * c["width"]
        if c["kind"] == "embed_fwd":
            return {"bytes": c["n"] * tb + (rows + _distinct(c["n"], c["vocab"]) * c["width"]) * es, "flops": rows}
        m = c["micro"]
        return {"bytes": m * (c["n"] * tb + rows * es) + c["vocab"] * c["width"] * 4, "flops": m * rows}
    if c["kind"].startswith("scan"):
        one = c["batch"] * c["length"] * c["channels"]
        part = c["batch"] * c["channels"] * 4 if c["state"] else 0
        if c["kind"] == "scan_fwd":
            return {"bytes": 3 * one * es + 2 * part, "flops": 10 * one}
        # the inputs and gates of the backward are those the forward read
        return {"bytes": 6 * one * es + 4 * part, "flops": 28 * one}
    rows = c["rows"] * c["classes"]
    return {"bytes": 2 * rows * es + c["rows"] * (c["top"] * (4 + es) + 8),
            "flops": rows * (12 if c["labels"] and c["tau"] != 1 else 7)}


def _exact_scan(s):
    c = s["case"]
    B, T, D = c["batch"], c["length"], c["channels"]
    z = lambda t: t.to(torch.float64)
    x, f = z(s["x"]).transpose(0, 1), torch.sigmoid(z(s["gate"])).transpose(0, 1)
    keep = torch.sigmoid(-z(s["gate"])).transpose(0, 1)
    live = torch.ones(T, B, 1, device=DEV, dtype=torch.bool)
    if s["lengths"] is not None:
        live = (torch.arange(T, device=DEV)[:, None] < s["lengths"])[..., None]
    state = torch.zeros(B, D, device=DEV, dtype=torch.float64) if s["h0"] is None else z(s["h0"])
    before = torch.empty(T, B, D, device=DEV, dtype=torch.float64)
    after = torch.empty_like(before)
    for t in range(T):
        before[t] = state
        state = torch.where(live[t], f[t] * state + keep[t] * x[t], state)
        after[t] = state
    out = [torch.where(live, after, 0.0).transpose(0, 1)] + ([state] if c["state"] else [])
    del after
    if c["kind"] == "scan_fwd":
        return out
    dh = z(s["dh"]).transpose(0, 1)
    carry = torch.zeros(B, D, device=DEV, dtype=torch.float64) if s["dhT"] is None else z(s["dhT"])
    G = torch.zeros_like(before)
    for t in range(T - 1, -1, -1):
        total = dh[t] + carry
        G[t] = torch.where(live[t], total, 0.0)
        carry = torch.where(live[t], f[t] * total, carry)
    out += [(G * keep).transpose(0, 1), (G * (before - x) * f * keep).transpose(0, 1)]
    return out + ([carry] if c["state"] else [])


def _exact_distill(s):
    c = s["case"]
    tau, alpha, n = c["tau"], c["alpha"], c["rows"]
    z = s["logits"].to(torch.float64)
    index, held = s["index"].long(), s["index"] >= 0
    t = s["teacher"].to(torch.float64) / tau
    t = t.masked_fill(~held, -math.inf)
    empty = ~held.any(1)
    t[empty] = 0.0
    logp = torch.log_softmax(t, 1)
    p = torch.where(held, torch.exp(logp), 0.0)
    logq = torch.log_softmax(z / tau, 1)
    r = torch.arange(n, device=DEV)[:, None].expand_as(index)
    picked = logq[r, index.clamp(min=0)]
    loss = alpha * tau ** 2 * torch.where(held, p * (logp - picked), 0.0).sum(1)
    d = alpha * tau * torch.exp(logq)
    del logq
    d[empty] = 0.0
    d.index_put_((r[held], index[held]), -alpha * tau * p[held], accumulate=True)
    if s["labels"] is not None:
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        y = s["labels"].long()[rows]
        logs = torch.log_softmax(z[rows], 1)
        k = torch.arange(len(rows), device=DEV)
        loss[rows] -= (1 - alpha) * logs[k, y]
        hard = torch.exp(logs)
        hard[k, y] -= 1.0
        d[rows] += (1 - alpha) * hard
    w = s["scale"] * (torch.ones(n, device=DEV, dtype=torch.float64) if s["weight"] is None
                      else s["weight"].to(torch.float64))
    return [loss, d * w[:, None]]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "embed_fwd":
        t = s["tokens"][0].long()
        out = torch.zeros(case["n"], case["width"], device=DEV, dtype=torch.float64)
        out[t >= 0] = s["table"].to(torch.float64)[t[t >= 0]] * s["scale"]
        return out
    if case["kind"] == "embed_bwd":
        total = torch.zeros(case["vocab"], case["width"], device=DEV, dtype=torch.float64)
        for t, dout in zip(s["tokens"], s["dout"]):
            t = t.long()
            total.index_put_((t[t >= 0],), dout.to(torch.float64)[t >= 0] * s["scale"], accumulate=True)
        return total
    return _exact_distill(s) if case["kind"] == "distill" else _exact_scan(s)
