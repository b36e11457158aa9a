"""The sequence operators' definitions in 64 bits on the CPU, each with an elementwise bound of the rounding
errors of an evaluation in 32 bits.

U is the unit roundoff of fp32; a value stored as bf16 adds 2^-8 of itself.  The bounds follow the sums: a sum
of n terms in any order is off by at most n U times the sum of their magnitudes; a chain h_t = f h_{t-1} + b by
E_t = f E_{t-1} + (magnitude at t) times U and the number of roundings of a step (a gate and its complement: an
exponential, a sum, a reciprocal, two products, at most 8 U together; the products and the sum of a step, and
of the same step once more where stretches are composed: 8 U)."""
import math

import torch

U = 2.0 ** -24
STORE = {"f32": U, "bf16": 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = 16 * U


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


def within(got, ref, bound, dtype):
    """Every element within bound + one rounding to dtype; NaN exactly where the reference has it."""
    got = f64(got)
    assert got.shape == ref.shape, (got.shape, ref.shape)
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), (int(torch.isnan(got).sum()), int(nan.sum()))
    err = torch.where(nan, 0.0, (got - ref).abs())
    lim = torch.where(nan, 0.0, bound * (1 + 2.0 ** -7) + STORE[dtype] * 1.01 * ref.abs() + 1e-37)
    worst = (err - lim).max().item() if err.numel() else 0.0
    assert worst <= 0.0, (worst, err.max().item(), (err / lim).max().item())


# ---- embedding ---------------------------------------------------------------------------------

def embed_fwd(table, tokens, scale):
    t = tokens.cpu().long()
    out = torch.zeros(len(t), table.shape[1], dtype=torch.float64)
    ok = (t >= 0) & (t < table.shape[0])
    out[ok] = f64(table)[t[ok]] * scale
    out[t >= table.shape[0]] = math.nan
    return out, U * out.abs()


def embed_bwd(vocab, tokens, dout, scale, old=None):
    t = tokens.cpu().long()
    ok = (t >= 0) & (t < vocab)
    d = f64(dout)[ok] * scale
    total = torch.zeros(vocab, d.shape[1], dtype=torch.float64)
    size = torch.zeros_like(total)
    total.index_add_(0, t[ok], d)
    size.index_add_(0, t[ok], d.abs())
    count = torch.bincount(t[ok], minlength=vocab).to(torch.float64)[:, None]
    bound = (count + 2) * U * size
    if old is not None:
        total = total + f64(old)
        bound = bound + 2 * U * torch.where(count > 0, f64(old).abs() + size, 0.0)
    return total, bound


# ---- recurrence --------------------------------------------------------------------------------

def scan(x, gate, lengths, h0, dh=None, dhT=None):
    """{name: (value, bound)} of h, hT and, given dh, of dx, dgate, dh0."""
    B, T, D = x.shape
    x, g = f64(x), f64(gate)
    f, keep = torch.sigmoid(g), torch.sigmoid(-g)
    n = torch.full((B,), T) if lengths is None else lengths.cpu().long().clamp(0, T)
    state = torch.zeros(B, D, dtype=torch.float64) if h0 is None else f64(h0)
    size, err = state.abs(), torch.zeros_like(state)
    h, before, bsize, berr, herr = (torch.zeros(B, T, D, dtype=torch.float64) for _ in range(5))
    for t in range(T):
        live = (t < n)[:, None]
        before[:, t], bsize[:, t], berr[:, t] = state, size, err
        b = keep[:, t] * x[:, t]
        new, nsize = f[:, t] * state + b, f[:, t] * size + b.abs()
        nerr = f[:, t] * err + STEP * nsize
        state, size, err = (torch.where(live, p, q) for p, q in ((new, state), (nsize, size), (nerr, err)))
        h[:, t], herr[:, t] = torch.where(live, state, 0.0), torch.where(live, err, 0.0)
    out = {"h": (h, herr), "hT": (state, err)}
    if dh is None:
        return out
    dh = f64(dh)
    c = torch.zeros(B, D, dtype=torch.float64) if dhT is None else f64(dhT)
    csize, cerr = c.abs(), torch.zeros_like(c)
    dx, dg, dxe, dge = (torch.zeros(B, T, D, dtype=torch.float64) for _ in range(4))
    for t in range(T - 1, -1, -1):
        live = (t < n)[:, None]
        G, gs = dh[:, t] + c, dh[:, t].abs() + csize
        ge = cerr + STEP * gs
        diff, ds = before[:, t] - x[:, t], bsize[:, t] + x[:, t].abs()
        fk = f[:, t] * keep[:, t]
        for o, v in ((dx, keep[:, t] * G), (dxe, keep[:, t] * (ge + STEP * gs)), (dg, G * diff * fk),
                     (dge, fk * (ge * ds + gs * (berr[:, t] + 2 * STEP * ds)))):
            o[:, t] = torch.where(live, v, 0.0)
        c, csize, cerr = (torch.where(live, p, q) for p, q in
                          ((f[:, t] * G, c), (f[:, t] * gs, csize), (f[:, t] * (ge + STEP * gs), cerr)))
    return {**out, "dx": (dx, dxe), "dgate": (dg, dge), "dh0": (c, cerr)}


# ---- distillation ------------------------------------------------------------------------------

def distill(z, index, teacher, labels, weight, tau, alpha, scale):
    """(loss, bound, dlogits, bound)"""
    n, V = z.shape
    z, t = f64(z), f64(teacher)
    loss, lb = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    d, db = torch.zeros(n, V, dtype=torch.float64), torch.zeros(n, V, dtype=torch.float64)
    for r in range(n):
        idx = index[r].cpu().long()
        y = -1 if labels is None else int(labels[r])
        w = scale * (1.0 if weight is None else float(weight[r]))
        if (idx >= V).any() or y >= V:
            loss[r], d[r] = math.nan, math.nan
            continue
        held = idx >= 0
        t_r = t[r][held] / tau
        if len(t_r) and not (t_r == -math.inf).all():
            lp, lq = torch.log_softmax(t_r, 0), torch.log_softmax(z[r] / tau, 0)
            p, q, picked = torch.exp(lp), torch.exp(lq), lq[idx[held]]
            on = p > 0
            p, lp, picked, i = p[on], lp[on], picked[on], idx[held][on]
            loss[r] += alpha * tau ** 2 * (p * (lp - picked)).sum()
            P = torch.zeros(V, dtype=torch.float64).index_add_(0, i, p)
            d[r] += alpha * tau * w * (q - P)
            far_q = torch.nan_to_num((z[r].max() - z[r]) / tau, posinf=0.0)
            far_t = ((t_r.max() - t_r) / tau)[on]
            # a sum of n terms, each an exponential of an argument with two roundings
            dq = U * (V + 8 + 2 * (q * far_q).sum())
            dt = U * (len(p) + 8 + 2 * (p * far_t).sum())
            terms = far_t + far_q[i] + 2 * (lp.abs() + picked.abs()) + 4
            lb[r] += abs(alpha) * tau ** 2 * ((p * (dq + dt + 8 * U * terms)).sum()
                                              + (p * (dt + U * (2 * far_t + 8)) * (lp - picked).abs()).sum())
            pe = torch.zeros(V, dtype=torch.float64).index_add_(0, i, p * (dt + U * (2 * far_t + 8 + len(p))))
            db[r] += abs(alpha * tau * w) * (q * (dq + U * (2 * far_q + 8)) + pe + 4 * U * P)
        if y >= 0:
            ls = torch.log_softmax(z[r], 0)
            s = torch.exp(ls)
            hot = torch.zeros(V, dtype=torch.float64)
            hot[y] = 1.0
            far = torch.nan_to_num(z[r].max() - z[r], posinf=0.0)
            ds = U * (V + 8 + 2 * (s * far).sum())
            loss[r] += (1 - alpha) * -ls[y]
            lb[r] += abs(1 - alpha) * (ds + 8 * U * (far[y] + ls[y].abs() + 4))
            d[r] += (1 - alpha) * w * (s - hot)
            db[r] += abs((1 - alpha) * w) * (s * (ds + U * (2 * far + 8)) + 4 * U * hot)
        lb[r] += 4 * U * loss[r].abs()
        db[r] += 8 * U * d[r].abs()
    return loss, lb, d, db
