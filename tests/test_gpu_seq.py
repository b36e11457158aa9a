"""The sequence operators on the GPU against their definitions in 64 bits (seq_ref), elementwise, at the sizes,
strides, masks and lengths where their kernels can go wrong; the space around every output stays as it was."""
import math

import pytest
import torch

from tests import seq_ref as R

pytestmark = pytest.mark.gpu

MARK = 77.0     # what the space around an output holds


def _seq():
    from paper_2103_08802_amd import seq
    return seq


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _stream():
    return torch.cuda.current_stream().cuda_stream


class Framed:
    """A tensor inside a larger buffer of MARKs: `lead` elements before it, rows (last dimension) `pad` apart."""

    def __init__(self, shape, dtype, lead=0, pad=0, fill=None):
        shape = tuple(shape)
        rows = math.prod(shape[:-1])
        w = shape[-1] + pad
        self.buf = torch.full((lead + rows * w + 64,), MARK, dtype=dtype, device="cuda")
        self.t = self.buf[lead:lead + rows * w].view(*shape[:-1], w)[..., :shape[-1]]
        if fill is not None:
            self.t.copy_(fill)

    def intact(self):
        inside = torch.zeros_like(self.buf, dtype=torch.bool)
        o = self.t.storage_offset()
        rows = math.prod(self.t.shape[:-1])
        w = self.t.stride(-2) if self.t.dim() > 1 and rows > 0 else self.t.shape[-1]
        inside[o:o + rows * w].view(rows, w)[:, :self.t.shape[-1]] = True
        assert bool((self.buf[~inside] == MARK).all())


# ---- embedding ---------------------------------------------------------------------------------

def _tokens(g, n, vocab, kind, dtype):
    if kind == "one":
        t = torch.full((n,), vocab - 1)
    elif kind == "none":
        t = torch.full((n,), -1)
    else:
        t = (torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * math.log(vocab + 1)) - 1).long().clamp(0, vocab - 1)
        if kind == "mixed":
            r = torch.rand(n, generator=g)
            t[r < 0.1] = -1
            t[(r > 0.1) & (r < 0.13)] = -9 if n % 2 else -(1 << 30)
            t[r > 0.97] = vocab
            t[r > 0.99] = (1 << 31) - 1
            if dtype is torch.int64:
                t[r > 0.995] = (1 << 40) + 1                 # low 32 bits: a row of the table
                t[(r > 0.13) & (r < 0.14)] = -(1 << 40) + 1
    return t.to(dtype)


EMBED = [
    # n, width, vocab, rows, table, tokens, kind, lead, pad
    (1, 1, 1, "f32", "f32", torch.int32, "plain", 0, 0),
    (1, 8, 5, "bf16", "bf16", torch.int64, "plain", 0, 0),
    (3, 16, 2, "bf16", "f32", torch.int64, "plain", 0, 8),       # fp32 table, bf16 rows
    (33, 7, 3, "f32", "bf16", torch.int32, "mixed", 1, 2),       # odd width, rows off 16 bytes
    (64, 24, 9, "bf16", "bf16", torch.int64, "one", 0, 0),       # one run over two tiles
    (65, 24, 9, "bf16", "bf16", torch.int64, "none", 0, 0),      # padding only
    (31, 2056, 7, "bf16", "bf16", torch.int32, "mixed", 8, 8),   # wider than a workgroup's pieces
    (257, 515, 40, "f32", "f32", torch.int64, "mixed", 3, 1),
    (2049, 40, 511, "bf16", "bf16", torch.int32, "mixed", 0, 0), # one radix pass, two workgroups
    (4100, 8, 512, "f32", "f32", torch.int64, "mixed", 0, 0),    # two passes
    (5000, 20, 70001, "bf16", "bf16", torch.int64, "mixed", 0, 4),
    (3000, 9, 300001, "f32", "f32", torch.int32, "mixed", 0, 0), # three passes
    (140001, 8, 513, "bf16", "bf16", torch.int64, "mixed", 0, 0),  # histograms summed by a launch of their own
    (20000, 8, 4, "f32", "f32", torch.int32, "plain", 0, 0),     # runs over hundreds of tiles
]


@pytest.mark.parametrize("n,width,vocab,rows,table,tok,kind,lead,pad", EMBED)
def test_embed(n, width, vocab, rows, table, tok, kind, lead, pad):
    seq = _seq()
    g = _gen(n * 7 + width)
    tokens = _tokens(g, n, vocab, kind, tok).cuda()
    tab = Framed((vocab, width), R.DT[table], lead, pad, torch.randn(vocab, width, generator=g))
    out = Framed((n, width), R.DT[rows], lead, pad)
    scale = 1.7
    d = seq.embed_desc(tab.t, tokens, out.t, scale)
    seq.pnn_embed_fwd(d, tab.t, tokens, out.t, _stream())
    R.within(out.t, *R.embed_fwd(tab.t, tokens, d.scale), rows)
    out.intact()
    # the gradient, then a second batch added to it
    dout = Framed((n, width), R.DT[rows], lead, pad, torch.randn(n, width, generator=g))
    grad = Framed((vocab, width), torch.float32, lead, pad, torch.full((vocab, width), 5.0))
    ws = torch.full((seq.pnn_embed_workspace_size(d),), 0xAB, dtype=torch.uint8, device="cuda")
    d = seq.embed_desc(grad.t, tokens, dout.t, scale)
    seq.pnn_embed_bwd(d, dout.t, tokens, grad.t, False, ws, _stream())
    first = grad.t.clone()
    R.within(first, *R.embed_bwd(vocab, tokens, dout.t, d.scale), "f32")
    seq.pnn_embed_bwd(d, dout.t, tokens, grad.t, True, ws, _stream())
    R.within(grad.t, *R.embed_bwd(vocab, tokens, dout.t, d.scale, first), "f32")
    grad.intact()
    # no sum depends on timing
    again = torch.empty(vocab, width, device="cuda")
    d = seq.embed_desc(again, tokens, dout.t, scale)
    ws.fill_(0x11)
    seq.pnn_embed_bwd(d, dout.t, tokens, again, False, ws, _stream())
    assert torch.equal(again, first)


def test_embed_empty():
    seq = _seq()
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    grad = torch.full((9, 5), 3.0, device="cuda")
    d = seq.embed_desc(grad, none, torch.empty(0, 5, device="cuda"), 2.0)
    seq.pnn_embed_fwd(d, grad, none, None, _stream())
    seq.pnn_embed_bwd(d, None, none, grad, True, None, _stream())
    assert bool((grad == 3.0).all())
    seq.pnn_embed_bwd(d, None, none, grad, False, None, _stream())
    assert bool((grad == 0.0).all())


def test_embed_values_outside_the_rows_used():
    """Infinities and NaN in the gradients of padding stay out; those of a token reach its row only."""
    seq = _seq()
    tokens = torch.tensor([2, -1, 0, 2, 5], dtype=torch.int32, device="cuda")
    dout = torch.ones(5, 8, device="cuda")
    dout[1], dout[4], dout[2, 3] = math.nan, math.inf, math.inf
    grad = torch.empty(4, 8, device="cuda")
    d = seq.embed_desc(grad, tokens, dout, 1.0)
    ws = torch.empty(seq.pnn_embed_workspace_size(d), dtype=torch.uint8, device="cuda")
    seq.pnn_embed_bwd(d, dout, tokens, grad, False, ws, _stream())
    want = torch.zeros(4, 8)
    want[0], want[2], want[0, 3] = 1.0, 2.0, math.inf
    assert torch.equal(grad.cpu(), want)


# ---- recurrence --------------------------------------------------------------------------------

SCAN = [
    # batch, length, channels, dtype, layout, lengths, state, lead
    (1, 1, 1, "f32", "dense", None, True, 0),
    (64, 1, 130, "bf16", "dense", None, True, 0),
    (3, 2, 64, "bf16", "halves", None, False, 0),
    (2, 7, 33, "f32", "halves", "ragged", True, 1),
    (5, 16, 128, "bf16", "time", "ragged", True, 0),
    (4, 17, 96, "f32", "dense", "ragged", True, 0),
    (2, 63, 257, "bf16", "halves", None, True, 1),
    (3, 128, 40, "bf16", "dense", "ragged", True, 0),
    (1, 129, 1024, "bf16", "dense", None, True, 0),
    (1, 256, 8, "f32", "time", None, False, 0),
    (2, 300, 70, "f32", "dense", "ragged", True, 0),
    (7, 511, 24, "bf16", "halves", "ragged", True, 0),
    (1, 1025, 65, "bf16", "dense", None, True, 0),
    (2, 1537, 66, "bf16", "time", "ragged", True, 0),
    (1, 5003, 9, "f32", "dense", None, True, 0),
    (100, 1500, 30, "bf16", "halves", "ragged", True, 0),        # several tiles for each of two workgroups
    (40, 2311, 66, "f32", "dense", "ragged", True, 0),           # two channel groups, three workgroups each
    (300, 40, 131, "bf16", "halves", "ragged", True, 1),         # pairs of an odd number of channels, rows on odd elements
    (260, 150, 66, "bf16", "time", "ragged", True, 0),
    (520, 300, 5, "f32", "dense", "ragged", True, 0),            # eight-wave tiles, several of them
    (600, 70, 65, "bf16", "dense", None, False, 0),
]


def _seq_tensors(shape, dtype, layout, lead, fills):
    """Tensors [batch][length][channels]: dense, pairs as the halves of one, or with the batch inside the steps."""
    B, T, D = shape
    if layout == "time":
        fr = [Framed((T, B, D), dtype, lead, 0, None if f is None else f.transpose(0, 1)) for f in fills]
        return fr, [f.t.transpose(0, 1) for f in fr]
    if layout == "halves" and len(fills) == 2:
        both = None if fills[0] is None else torch.cat(fills, 2)
        f = Framed((B, T, 2 * D), dtype, lead, 0, both)
        return [f], [f.t[..., :D], f.t[..., D:]]
    fr = [Framed(shape, dtype, lead, 0, f) for f in fills]
    return fr, [f.t for f in fr]


@pytest.mark.parametrize("B,T,D,dtype,layout,lens,state,lead", SCAN)
def test_scan(B, T, D, dtype, layout, lens, state, lead):
    seq = _seq()
    g = _gen(B * 1000 + T * 10 + D)
    dt, shape = R.DT[dtype], (B, T, D)
    gate = torch.randn(shape, generator=g) + torch.rand(D, generator=g) * 10 - 3
    gate[0, 0, 0], gate[0, -1, -1] = 95.0, -95.0                       # closed and open to the last bit
    rnd = lambda: torch.randn(shape, generator=g)
    _, (x, gt) = _seq_tensors(shape, dt, layout, lead, [rnd(), gate])
    _, (dh,) = _seq_tensors(shape, dt, layout, lead, [rnd()])
    fh, (h,) = _seq_tensors(shape, dt, layout, lead, [None])
    fg, (dx, dg) = _seq_tensors(shape, dt, layout, lead, [None, None])
    lengths = None
    if lens:
        lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        lengths[0], lengths[-1] = T + 9, 0
        if B > 2:
            lengths[1] = -3
        lengths = lengths.cuda()
        # what stands behind a sequence's end is not part of it
        for b in range(B):
            n = max(0, min(T, int(lengths[b])))
            x[b, n:], gt[b, n:], dh[b, n:] = math.nan, math.inf, math.nan
    vec = lambda: torch.randn(B, D, generator=g).cuda()
    h0, dhT = (vec(), vec()) if state else (None, None)
    hT, dh0 = (Framed((B, D), torch.float32, 1) for _ in range(2))
    d = seq.scan_desc(x, gt, h, dh, dx, dg)
    n_states, n_ws = seq.pnn_scan_sizes(d)
    states = torch.full((n_states // 4 + 8,), MARK, device="cuda")
    ws = torch.full((n_ws + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    seq.pnn_scan_fwd(d, x, gt, lengths, h0, h, hT.t, states, ws, _stream())
    assert bool((states[n_states // 4:] == MARK).all()) and bool((ws[n_ws:] == 0xAB).all())
    seq.pnn_scan_bwd(d, x, gt, lengths, states, dh, dhT, dx, dg, dh0.t, ws, _stream())
    ref = R.scan(x, gt, lengths, h0, dh, dhT)
    for name, t, ty in (("h", h, dtype), ("hT", hT.t, "f32"), ("dx", dx, dtype), ("dgate", dg, dtype),
                        ("dh0", dh0.t, "f32")):
        R.within(t, *ref[name], ty)
    for f in fh + fg + [hT, dh0]:
        f.intact()
    # without what is optional: the same h; the state in place of the first one
    h2 = torch.empty(shape, dtype=dt, device="cuda")
    d2 = seq.scan_desc(x, gt, h2)
    ws.fill_(0x11)
    place = h0.clone() if state else None
    seq.pnn_scan_fwd(d2, x, gt, lengths, place, h2, place, None, ws, _stream())
    assert torch.equal(h2, h.contiguous())
    if state:
        assert torch.equal(place, hT.t)
    dx1, dg1 = dx.clone(), dg.clone()
    place = dhT.clone() if state else None
    seq.pnn_scan_bwd(d, x, gt, lengths, states, dh, place, dx, dg, place, ws, _stream())
    assert torch.equal(dx, dx1) and torch.equal(dg, dg1)
    if state:
        assert torch.equal(place, dh0.t)


def test_scans_side_by_side():
    """Sequences whose tiles are dealt to every compute unit, on three streams at once: the bits each gives alone."""
    seq = _seq()
    g = _gen(21)
    B, T, D = 1, 9001, 200
    runs = []
    for i in range(3):
        x, dh = (torch.randn(B, T, D, generator=g).cuda() for _ in range(2))
        gate = (torch.randn(B, T, D, generator=g) + torch.rand(D, generator=g) * 8 - 2).cuda()
        h, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        d = seq.scan_desc(x, gate, h, dh, dx, dg)
        n, w = seq.pnn_scan_sizes(d)
        states, ws = torch.empty(n // 4, device="cuda"), torch.empty(w, dtype=torch.uint8, device="cuda")
        runs.append((d, x, gate, h, dh, dx, dg, states, ws, torch.cuda.Stream()))

    def go(r):
        d, x, gate, h, dh, dx, dg, states, ws, _ = r
        seq.pnn_scan_fwd(d, x, gate, None, None, h, None, states, ws, _stream())
        seq.pnn_scan_bwd(d, x, gate, None, states, dh, None, dx, dg, None, ws, _stream())

    alone = []
    for r in runs:
        go(r)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (r[3], r[5], r[6])])
    for _ in range(5):
        for r in runs:
            with torch.cuda.stream(r[-1]):
                go(r)
    torch.cuda.synchronize()
    for r, want in zip(runs, alone):
        for a, b in zip((r[3], r[5], r[6]), want):
            assert torch.equal(a, b)


def test_scan_step_by_step_is_the_sequence():
    """Single steps with the state in place give the states of the whole sequence, up to the roundings of either."""
    seq = _seq()
    B, T, D = 3, 40, 72
    g = _gen(5)
    x = torch.randn(B, T, D, generator=g).cuda()
    gate = (torch.randn(B, T, D, generator=g) * 2).cuda()
    h = torch.empty_like(x)
    d = seq.scan_desc(x, gate, h)
    ws = torch.empty(seq.pnn_scan_sizes(d)[1] + 256, dtype=torch.uint8, device="cuda")
    seq.pnn_scan_fwd(d, x, gate, None, None, h, None, None, ws, _stream())
    ref, bound = R.scan(x, gate, None, None)["h"]
    state = torch.zeros(B, D, device="cuda")
    one = torch.empty(B, 1, D, device="cuda")
    for t in range(T):
        xt, gt = x[:, t:t + 1], gate[:, t:t + 1]
        seq.pnn_scan_fwd(seq.scan_desc(xt, gt, one), xt, gt, None, state, one, state, None, None, _stream())
        R.within(one[:, 0], ref[:, t], bound[:, t], "f32")
    R.within(h, ref, bound, "f32")


def test_scan_empty():
    seq = _seq()
    e = torch.empty(2, 0, 5, device="cuda")
    d = seq.scan_desc(e, e, e, e, e, e)
    a, b = torch.arange(10.0, device="cuda").view(2, 5), torch.zeros(2, 5, device="cuda")
    seq.pnn_scan_fwd(d, None, None, None, a, None, b, None, None, _stream())
    assert torch.equal(a, b)
    seq.pnn_scan_fwd(d, None, None, None, None, None, b, None, None, _stream())
    assert not b.any()
    seq.pnn_scan_bwd(d, None, None, None, None, None, a, None, None, b, None, _stream())
    assert torch.equal(a, b)


def test_scan_gradient_is_the_difference_quotient():
    """dL/dx and dL/dgate of L = sum(dh h) + sum(dhT hT) against central differences of the 64-bit definition."""
    seq = _seq()
    B, T, D = 2, 19, 3
    g = _gen(11)
    x, gate, dh = (torch.randn(B, T, D, generator=g) for _ in range(3))
    h0, dhT = torch.randn(B, D, generator=g), torch.randn(B, D, generator=g)
    lengths = torch.tensor([19, 13], dtype=torch.int32)
    xs, gs, ds = x.cuda(), gate.cuda(), dh.cuda()
    h, dx, dg, dh0 = torch.empty_like(xs), torch.empty_like(xs), torch.empty_like(xs), torch.empty(B, D, device="cuda")
    d = seq.scan_desc(xs, gs, h, ds, dx, dg)
    n, w = seq.pnn_scan_sizes(d)
    states, ws = torch.empty(n // 4, device="cuda"), torch.empty(w + 256, dtype=torch.uint8, device="cuda")
    seq.pnn_scan_fwd(d, xs, gs, lengths.cuda(), h0.cuda(), h, None, states, ws, _stream())
    seq.pnn_scan_bwd(d, xs, gs, lengths.cuda(), states, ds, dhT.cuda(), dx, dg, dh0, ws, _stream())

    def loss(x, gate, h0):
        r = R.scan(x, gate, lengths, h0)
        return float((r["h"][0] * dh.double()).sum() + (r["hT"][0] * dhT.double()).sum())

    eps = 1e-5                                        # truncation eps^2, cancellation 1e-16 / eps: 1e-9 in all
    args = [x.double(), gate.double(), h0.double()]
    for k, got in ((0, dx), (1, dg), (2, dh0)):
        flat = args[k].view(-1)
        for i in range(0, flat.numel(), 5):
            v = flat[i].item()
            flat[i] = v + eps
            up = loss(*args)
            flat[i] = v - eps
            down = loss(*args)
            flat[i] = v
            assert abs((up - down) / (2 * eps) - got.view(-1)[i].item()) <= 2e-5, (k, i)


# ---- distillation ------------------------------------------------------------------------------

DISTILL = [
    # rows, classes, top, logits, teacher, tau, alpha, labels, masked, lead, pad
    (1, 1, 1, "f32", "f32", 1.0, 0.5, True, False, 0, 0),
    (3, 2, 2, "bf16", "f32", 2.0, 0.5, True, False, 0, 0),
    (5, 10, 0, "f32", "f32", 1.0, 0.5, True, False, 0, 0),             # labels only
    (6, 100, 5, "bf16", "bf16", 4.0, 1.0, False, False, 0, 4),         # teacher only
    (9, 63, 63, "f32", "bf16", 1.0, 0.9, True, True, 1, 0),
    (9, 64, 20, "f32", "f32", 0.5, 0.3, True, True, 0, 0),
    (17, 200, 7, "bf16", "bf16", 2.0, 0.5, True, True, 3, 5),          # rows off 16 bytes
    (12, 1000, 10, "f32", "f32", 1.0, 0.5, True, True, 0, 0),
    (11, 1001, 64, "bf16", "f32", 3.0, 0.7, True, True, 1, 0),
    (4, 2049, 300, "bf16", "bf16", 2.0, 0.5, True, True, 0, 7),
    (3, 4097, 1024, "f32", "f32", 1.0, 0.5, True, True, 0, 0),
    (3, 16391, 33, "bf16", "bf16", 2.0, 0.5, True, True, 5, 1),
    (2, 32768, 16, "f32", "f32", 2.0, 0.5, True, True, 0, 0),
    (3, 65551, 64, "bf16", "bf16", 2.0, 0.5, True, True, 0, 1),
    (2, 70000, 64, "f32", "bf16", 1.0, 0.9, True, True, 0, 0),
    (2, 140003, 50, "bf16", "f32", 4.0, 0.5, True, True, 0, 0),
]


def _distill_inputs(g, n, V, k, masked):
    z = torch.randn(n, V, generator=g) * 3
    index = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(n)]) if k else torch.zeros(n, 0, dtype=torch.long)
    teacher = torch.randn(n, k, generator=g) * 3
    labels = torch.randint(0, V, (n,), generator=g)
    if masked:
        index[torch.rand(n, k, generator=g) < 0.2] = -1
        if k > 1:
            index[:, 1] = torch.where(torch.rand(n, generator=g) < 0.5, index[:, 0], index[:, 1])   # a class twice
        labels[torch.rand(n, generator=g) < 0.3] = -1
        index[0] = -1                                                   # no entry
        if n > 2:
            index[1], labels[1] = -5, -1                                # nothing at all
        if n > 3:
            teacher[3, ::2] = -math.inf                                 # entries without mass
        if n > 4:
            teacher[4] = -math.inf
        if n > 5:
            z[5, torch.rand(V, generator=g) < 0.5] = torch.finfo(torch.bfloat16).min
            z[5, index[5].clamp(min=0)], z[5, labels[5].clamp(min=0)] = 0.5, -0.5
        if n > 6:
            z[6, torch.rand(V, generator=g) < 0.5] = -math.inf          # classes masked out
            z[6, index[6].clamp(min=0)], z[6, labels[6].clamp(min=0)] = 0.5, -0.5
        if n > 7:
            labels[7] = V
        if n > 8:
            index[8, -1] = V + 3
        if n > 10:
            labels[10] = max(int(index[10, 0]), 0)
    return z, index.to(torch.int32), teacher, labels.to(torch.int32)


@pytest.mark.parametrize("n,V,k,dtype,td,tau,alpha,labelled,masked,lead,pad", DISTILL)
def test_distill(n, V, k, dtype, td, tau, alpha, labelled, masked, lead, pad):
    seq = _seq()
    g = _gen(V + k)
    z, index, teacher, labels = _distill_inputs(g, n, V, k, masked)
    zf = Framed((n, V), R.DT[dtype], lead, pad, z)
    tf = Framed((n, k), R.DT[td], 0, 0, teacher)
    idx = index.cuda()
    labels = labels.cuda() if labelled else None
    weight = (torch.rand(n, generator=g) + 0.5).cuda() if masked else None
    loss, dz = torch.full((n + 1,), MARK, device="cuda"), Framed((n, V), R.DT[dtype], lead, pad)
    d = seq.distill_desc(zf.t, tf.t, dz.t, tau, alpha, 0.25)
    call = lambda z, l, dz, d=d: seq.pnn_distill_fwd_bwd(d, z, idx, tf.t, labels, weight, l, dz, _stream())
    call(zf.t, loss, dz.t)
    want = R.distill(zf.t, idx, tf.t, labels, weight, d.temperature, d.alpha, d.scale)
    R.within(loss[:n], want[0], want[1], "f32")
    R.within(dz.t, want[2], want[3], dtype)
    assert loss[n] == MARK
    dz.intact()
    # the loss alone, and the gradient in the logits' place: the same bits
    bits = lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
    only = torch.empty(n, device="cuda")
    call(zf.t, only, None)
    assert torch.equal(bits(only), bits(loss[:n]))
    call(zf.t, only, zf.t)
    assert torch.equal(bits(only), bits(loss[:n])) and torch.equal(bits(zf.t), bits(dz.t))
    zf.intact()


def test_distill_rows_without_terms_ignore_their_logits():
    seq = _seq()
    z = torch.full((3, 40), math.nan, device="cuda")
    z[2] = math.inf
    index = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    teacher = torch.full((3, 4), math.nan, device="cuda")
    labels = torch.full((3,), -1, dtype=torch.int32, device="cuda")
    loss, dz = torch.empty(3, device="cuda"), torch.empty_like(z)
    d = seq.distill_desc(z, teacher, dz, 2.0, 0.5, 1.0)
    seq.pnn_distill_fwd_bwd(d, z, index, teacher, labels, None, loss, dz, _stream())
    assert not loss.any() and not dz.any()
    # and one whose only class is masked out has no distribution
    labels[0] = 3
    z[0] = -math.inf
    seq.pnn_distill_fwd_bwd(d, z, index, teacher, labels, None, loss, dz, _stream())
    assert math.isnan(loss[0]) and bool(torch.isnan(dz[0]).all()) and not dz[1:].any()


@pytest.mark.parametrize("V", [50, 9000, 140003])          # one wave, a workgroup, a row read twice
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 4.0, 3.0])
def test_distill_rows_of_huge_logits(V, dtype, tau):
    """Rows whose logits are all the type's lowest value are uniform; huge ones of any sign keep their differences."""
    seq = _seq()
    g = _gen(V)
    low = torch.finfo(R.DT[dtype]).min
    z = torch.randn(6, V, generator=g)
    z[0] = low
    z[1] = -low / 4
    z[2] += 1e6
    z[3] *= 1e30
    z[4], z[4, 7] = low, 0.25
    z[5, ::2] = low
    index = torch.randint(0, V // 2, (6, 4), generator=g, dtype=torch.int32) * 2 + 1
    labels = index[:, 1].clone()
    index[3], labels[3] = z[3].argmax().item(), z[3].argmax().item()
    index[4], labels[4] = 7, 7
    teacher = torch.randn(6, 4, generator=g)
    zs = z.cuda().to(R.DT[dtype])
    loss, dz = torch.empty(6, device="cuda"), torch.empty_like(zs)
    d = seq.distill_desc(zs, teacher.cuda(), dz, tau, 0.5, 1.0)
    seq.pnn_distill_fwd_bwd(d, zs, index.cuda(), teacher.cuda(), labels.cuda(), None, loss, dz, _stream())
    want = R.distill(zs, index, teacher, labels, None, d.temperature, d.alpha, 1.0)
    R.within(loss, want[0], want[1], "f32")
    R.within(dz, want[2], want[3], dtype)


def test_distill_gradient_is_the_difference_quotient():
    seq = _seq()
    g = _gen(3)
    n, V, k = 3, 21, 5
    z, index, teacher, labels = _distill_inputs(g, n, V, k, False)
    labels[1] = -1
    index[2, 0] = index[2, 1]
    zs, dz, loss = z.cuda(), torch.empty(n, V, device="cuda"), torch.empty(n, device="cuda")
    d = seq.distill_desc(zs, teacher.cuda(), dz, 2.5, 0.6, 1.0)
    seq.pnn_distill_fwd_bwd(d, zs, index.cuda(), teacher.cuda(), labels.cuda(), None, loss, dz, _stream())
    total = lambda z: R.distill(z, index, teacher, labels, None, d.temperature, d.alpha, 1.0)[0].sum().item()
    eps, z64 = 1e-5, z.double()
    for i in range(n * V):
        f = z64.view(-1)
        v = f[i].item()
        f[i] = v + eps
        up = total(z64)
        f[i] = v - eps
        down = total(z64)
        f[i] = v
        assert abs((up - down) / (2 * eps) - dz.view(-1)[i].item()) <= 1e-5, i


# ---- streams and graphs ------------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    """All operators in a row on a stream of their own, then captured once and replayed on new inputs: every replay
    gives the bits of the eager calls."""
    seq = _seq()
    g = _gen(9)
    n, B, T, D, V, k = 600, 3, 200, 40, 300, 6
    table = torch.randn(V, 2 * D, generator=g).cuda()
    tokens = torch.zeros(B * T, dtype=torch.int64, device="cuda")
    rows, drows = torch.empty(B, T, 2 * D, device="cuda"), torch.empty(B, T, 2 * D, device="cuda")
    x, gate, dx, dg = rows[..., :D], rows[..., D:], drows[..., :D], drows[..., D:]
    h, dh = torch.empty(B, T, D, device="cuda"), torch.empty(B, T, D, device="cuda")
    loss = torch.empty(n, device="cuda")
    index = torch.randint(0, D, (n, k), generator=g, dtype=torch.int32).cuda()
    teacher = torch.randn(n, k, generator=g).cuda()
    grad = torch.empty_like(table)
    de = seq.embed_desc(table, tokens, rows.view(n, 2 * D), 2.0)
    ds = seq.scan_desc(x, gate, h, dh, dx, dg)
    dd = seq.distill_desc(h.view(n, D), teacher, dh.view(n, D), 2.0, 1.0, 1.0 / n)
    ns, nw = seq.pnn_scan_sizes(ds)
    states = torch.empty(ns // 4, device="cuda")
    ws = torch.empty(max(nw, seq.pnn_embed_workspace_size(de)) + 256, dtype=torch.uint8, device="cuda")

    def step():
        s = _stream()
        seq.pnn_embed_fwd(de, table, tokens, rows, s)
        seq.pnn_scan_fwd(ds, x, gate, None, None, h, None, states, ws, s)
        seq.pnn_distill_fwd_bwd(dd, h, index, teacher, None, None, loss, dh, s)
        seq.pnn_scan_bwd(ds, x, gate, None, states, dh, None, dx, dg, None, ws, s)
        seq.pnn_embed_bwd(de, drows, tokens, grad, False, ws, s)

    def result():
        torch.cuda.synchronize()
        return [t.clone() for t in (h, loss, drows, grad)]

    inputs = [torch.randint(-1, V, (B * T,), generator=g).cuda() for _ in range(3)]
    want = []
    side = torch.cuda.Stream()
    for t in inputs:
        tokens.copy_(t)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        want.append(result())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (2, 0, 1, 0):
        tokens.copy_(inputs[i])
        ws.fill_(i)
        graph.replay()
        for a, b in zip(result(), want[i]):
            assert torch.equal(a, b)
