"""Linear attention, norms and the policy loss in 64 bits on the CPU, each with an elementwise bound of the rounding
errors of an evaluation in 32 bits (as seq_ref, whose U, STORE and within serve here too).

A sum of n terms in any order is off by at most n U times the sum of their magnitudes; products on the matrix units are
counted with 2 U a term, whichever way their partial sums are rounded.  lambda^n = 2^(n log2 lambda), log2 lambda and
the product with n rounded once each, is off by 2 U n |ln lambda| of itself and an exponential's 2 U."""
import math

import torch

from tests.seq_ref import STORE, U, f64

BF = 2.0 ** -8     # a rounding to bf16


# ---- linear attention --------------------------------------------------------------------------

def _weights(d, T, n, shift=0):
    """lambda^(t - s) for s <= t < n, else 0, and its relative error in U, [T][T]"""
    t = torch.arange(T, dtype=torch.float64)
    apart = t[:, None] - t
    on = (apart >= 0) & (t[:, None] < n) & (t < n)
    w = torch.where(on, torch.exp(d * apart.clamp(min=0)), 0.0)
    w = torch.where(on & (apart == 0), 1.0, w)                      # 0^0
    far = torch.where(on & (apart > 0) & torch.isfinite(d), apart * d.abs(), 0.0)
    return w, 2 * far + 4


def _power(d, e):
    """lambda^e (0^0 = 1) and its relative error in U"""
    w = torch.where(e == 0, 1.0, torch.exp(d * e.clamp(min=1)))
    return w, torch.where((e > 0) & torch.isfinite(d), 2 * e * d.abs(), 0.0) + 4


def linattn(q, k, v, decay, lengths, s0, scale, dtype, dout=None, dsT=None):
    """{name: (value, bound)} of o, sT and, given dout, of dq, dk, dv, ds0"""
    B, T, H, K = q.shape
    kv, V = k.shape[2], v.shape[3]
    G = H // kv
    q, k, v, decay, s0, dout, dsT = (f64(t) for t in (q, k, v, decay, s0, dout, dsT))
    n = torch.full((B,), T) if lengths is None else lengths.cpu().long().clamp(0, T)
    names = ["o", "sT"] + (["dq", "dk", "dv", "ds0"] if dout is not None else [])
    shape = {"o": (B, T, H, V), "sT": (B, H, K, V), "dq": (B, T, H, K), "dk": (B, T, kv, K), "dv": (B, T, kv, V),
             "ds0": (B, H, K, V)}
    val = {x: torch.zeros(shape[x], dtype=torch.float64) for x in names}
    bnd = {x: torch.zeros(shape[x], dtype=torch.float64) for x in names}
    # an output's roundings on the way: the sums over widths, a chunk and the chunks, and for bf16 one operand of every
    # product and the split of the weighted values
    sums = 2 * U * (K + V + T + 64)
    way = sums + (BF * (1 + 2 ** -6) + 2 ** -16 if dtype == "bf16" else 0.0)
    z = torch.zeros(K, V, dtype=torch.float64)
    t = torch.arange(T, dtype=torch.float64)

    def add(name, at, value, size, rel):
        val[name][at] += value
        bnd[name][at] += size * rel

    for b in range(B):
        N = int(n[b])
        for h in range(H):
            g, d = h // G, decay[h]
            W, WE = _weights(d, T, N)
            Q, A, X = q[b, :, h], k[b, :, g], v[b, :, g]
            live = (t < N).to(torch.float64)[:, None]
            Q, A, X = (torch.where(live > 0, m, 0.0) for m in (Q, A, X))
            S0 = z if s0 is None else s0[b, h]
            since, se = _power(d, t + 1)
            until, ue = _power(d, (N - 1 - t).clamp(min=0))
            since, until = since[:, None] * live, until[:, None] * live
            se, ue = se[:, None], ue[:, None]
            whole, we = _power(d, torch.tensor(float(N), dtype=torch.float64))

            def causal(a, c, x, W=W, WE=WE):
                """sum over s of W[t][s] (a_t c_s) x_s and the magnitudes of its terms, with their weights' errors"""
                m = (a.abs() @ c.abs().t()) * W
                return ((a @ c.t()) * W) @ x, m @ x.abs(), U * ((m * WE) @ x.abs())

            o, m, e = causal(Q, A, X)
            add("o", (b, slice(None), h), scale * (o + since * (Q @ S0)),
                abs(scale) * (m + since * (Q.abs() @ S0.abs())), way)
            bnd["o"][b, :, h] += abs(scale) * (e + U * se * since * (Q.abs() @ S0.abs()))
            add("sT", (b, h), whole * S0 + (A * until).t() @ X,
                whole * S0.abs() + (A.abs() * until).t() @ X.abs(), sums)
            bnd["sT"][b, h] += U * (we * whole * S0.abs() + (A.abs() * until * ue).t() @ X.abs())
            if dout is None:
                continue
            D = torch.where(live > 0, dout[b, :, h], 0.0)
            Z = z if dsT is None else dsT[b, h]
            r, m, e = causal(D, X, A)
            add("dq", (b, slice(None), h), scale * (r + since * (D @ S0.t())),
                abs(scale) * (m + since * (D.abs() @ S0.abs().t())), way)
            bnd["dq"][b, :, h] += abs(scale) * (e + U * se * since * (D.abs() @ S0.abs().t()))
            Wt, WEt = W.t(), WE.t()
            for name, a, c, x, zz in (("dk", X, D, Q, Z.t()), ("dv", A, Q, D, Z)):
                r, m, e = causal(a, c, x, Wt, WEt)
                add(name, (b, slice(None), g), scale * r + until * (a @ zz),
                    abs(scale) * m + until * (a.abs() @ zz.abs()), way + G * U)
                bnd[name][b, :, g] += abs(scale) * e + U * ue * until * (a.abs() @ zz.abs())
            add("ds0", (b, h), whole * Z + scale * (Q * since).t() @ D,
                whole * Z.abs() + abs(scale) * (Q.abs() * since).t() @ D.abs(), sums)
            bnd["ds0"][b, h] += U * (we * whole * Z.abs() + abs(scale) * (Q.abs() * since * se).t() @ D.abs())
    return {x: (val[x], bnd[x]) for x in names}


# ---- norms -------------------------------------------------------------------------------------

ADDS = 40      # additions that a term of a row's sum passes: 16 in a lane, 6 over a wave, 16 waves
ROOT = ADDS / 2 + 4


def _rms(u, eps, err=None):
    """1 / sqrt(mean u^2 + eps) and its relative error, for u off by err"""
    r = 1 / torch.sqrt((u * u).mean(-1, keepdim=True) + eps)
    rel = torch.full_like(r, ROOT * U)
    if err is not None:
        rel = rel + (u.abs() * err).mean(-1, keepdim=True) * r * r
    return r, rel


def _gate(g):
    """sigmoid, silu and its slope with their errors (relative, absolute, absolute)"""
    s = torch.sigmoid(g)
    rel = U * (2 * g.abs() * (1 - s) + 6)
    far = torch.isinf(g)
    g0 = torch.where(far, 0.0, g)
    silu = torch.where(g == -math.inf, 0.0, g * s)
    slope = torch.where(far, s, s * (1 + g0 * (1 - s)))
    rel = torch.where(far, 0.0, rel)
    eslope = rel * slope.abs() + s * g0.abs() * (s * rel + 2 * U) + 4 * U * s * (1 + g0.abs() * (1 - s))
    return rel, silu, (rel + U) * silu.abs(), slope, eslope


def norm_fwd(x, w_post, gate, res, w_pre, post, pre, eps, alpha):
    """{name: (value, bound)} of h and y, inputs [..][width]"""
    x, w_post, gate, res, w_pre = (f64(t) for t in (x, w_post, gate, res, w_pre))
    a, rel = x, 0.0
    if post:
        r, rel = _rms(x, eps)
        a = x * r * (1.0 if w_post is None else w_post)
        rel = rel + 3 * U
    err = a.abs() * rel
    if gate is not None:
        grel, silu, esilu, _, _ = _gate(gate)
        err = err * silu.abs() + a.abs() * esilu + U * (a * silu).abs()
        a = a * silu
    h = alpha * a + (0.0 if res is None else res)
    err = abs(alpha) * (err + U * a.abs()) + U * h.abs()
    out = {"h": (h, err)}
    if pre:
        r, rel = _rms(h, eps, err)
        w = 1.0 if w_pre is None else w_pre
        y = h * r * w
        out["y"] = (y, y.abs() * (rel + 3 * U) + (err * r * w).abs())
    return out


def norm_bwd(x, w_post, gate, res, w_pre, dy, dh, post, pre, eps, alpha):
    """{name: (value, bound)} of dres, dx, dgate, dw_post, dw_pre"""
    x, w_post, gate, res, w_pre, dy, dh = (f64(t) for t in (x, w_post, gate, res, w_pre, dy, dh))
    out = {}
    h, eh = norm_fwd(x, w_post, gate, res, w_pre, post, False, eps, alpha)["h"]
    d = torch.zeros_like(x) if dh is None else dh
    W = d.shape[-1]
    count = d.numel() // W + ADDS
    total = lambda t: t.reshape(-1, W).sum(0)

    def back(u, eu, t, et):
        """r (t - u r^2 mean(t u)) and its error, for u and t off by eu and et"""
        r, rel = _rms(u, eps, eu)
        m = (t * u).mean(-1, keepdim=True) * r * r
        em = ((t * u).abs().mean(-1, keepdim=True) * (ADDS + 2) * U +
              (et * u.abs() + eu * t.abs()).mean(-1, keepdim=True)) * r * r
        em = em + m.abs() * (2 * rel + 4 * U)
        return r * (t - u * m), r * (et + u.abs() * em + eu * m.abs() + (t.abs() + (u * m).abs()) * (rel + 4 * U))

    err = U * d.abs()
    if pre:
        t = dy * (1.0 if w_pre is None else w_pre)
        v, e = back(h, eh, t, U * t.abs())
        r, rel = _rms(h, eps, eh)
        d, err = d + v, err + e + U * (d + v).abs()
        size = dy * h * r
        out["dw_pre"] = (total(size), total(size.abs() * (rel + 3 * U) + (dy * eh * r).abs()) +
                         count * U * total(size.abs()))
    out["dres"] = (d, err)
    d, err = alpha * d, abs(alpha) * err + U * (alpha * d).abs()
    n, rn = x, 0.0
    if post:
        r, rel = _rms(x, eps)
        n, rn = x * r * (1.0 if w_post is None else w_post), rel + 3 * U
    if gate is not None:
        grel, silu, esilu, slope, eslope = _gate(gate)
        v = d * n * slope
        out["dgate"] = (v, (err * n * slope).abs() + v.abs() * (rn + 3 * U) + (d * n).abs() * eslope)
        d, err = d * silu, err * silu.abs() + d.abs() * esilu + U * (d * silu).abs()
    if post:
        size = d * x * r
        out["dw_post"] = (total(size), total(size.abs() * (rel + 3 * U) + (err * x * r).abs()) +
                          count * U * total(size.abs()))
        t = d * (1.0 if w_post is None else w_post)
        d, err = back(x, torch.zeros_like(x), t, U * t.abs() + err * (1.0 if w_post is None else w_post.abs()))
    out["dx"] = (d, err)
    return out


# ---- policy loss -------------------------------------------------------------------------------

EXPS = 160     # additions that a term of a row's sum of exponentials passes: 128 in a thread, 6 over a wave, 16 waves


def policy(z, tokens, advantage, old, ref, weight, tau, low, high, kl, scale):
    """{name: (value, bound)} of loss, logp, dlogits (rows at a clip's border are not told apart)"""
    n, V = z.shape
    z, A, old, ref, weight = (f64(t) for t in (z, advantage, old, ref, weight))
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)
    val = {"loss": zero(n), "logp": zero(n), "dlogits": zero(n, V)}
    bnd = {x: torch.zeros_like(t) for x, t in val.items()}
    for r in range(n):
        a = int(tokens[r])
        if a < 0:
            continue
        if a >= V or (z[r] == -math.inf).all() or torch.isnan(z[r]).any() or (z[r] == math.inf).any():
            for t in val.values():
                t[r] = math.nan
            continue
        m = z[r].max()
        lp = torch.log_softmax(z[r] / tau, 0)
        p = torch.exp(lp)
        far = torch.nan_to_num((m - z[r]) / tau, posinf=0.0)
        l = lp[a]
        ds = U * (EXPS + 4 + 3 * (p * far).sum())
        logs = -(m / tau - torch.logsumexp(z[r] / tau, 0))
        el = ds + U * (3 * far[a] + 3 * logs.abs() + 2 * l.abs() + 2) if l != -math.inf else zero(())
        ratio, er = torch.ones((), dtype=torch.float64), zero(())
        if old is not None:
            ratio = torch.exp(l - old[r])
            er = ratio * (el + U * ((l - old[r]).abs() + 4)) if ratio > 0 else zero(())
        whole, cut = ratio * A[r], ratio.clamp(1 - low, 1 + high) * A[r]
        loss, c = (-cut, zero(())) if whole > cut else (-whole, -whole)
        e = A[r].abs() * er + 4 * U * loss.abs()
        ec = A[r].abs() * er + 2 * U * c.abs()
        if kl != 0:
            x = ref[r] - l
            up = torch.expm1(x)
            ex = el + U * x.abs()
            loss = loss + kl * (up - x)
            c = c - kl * up
            e = e + abs(kl) * (up.abs() * ex + 4 * U * (up.abs() + x.abs()))
            ec = ec + abs(kl) * ((up + 1) * ex + 4 * U * up.abs())
        e, ec = e + 4 * U * loss.abs(), ec + 2 * U * c.abs()
        w = scale / tau * (1.0 if weight is None else weight[r])
        hot = torch.zeros(V, dtype=torch.float64)
        hot[a] = 1.0
        val["loss"][r], bnd["loss"][r] = loss, e
        val["logp"][r], bnd["logp"][r] = l, el
        val["dlogits"][r] = w * c * (hot - p)
        g = abs(w) * (ec + 8 * U * c.abs())
        bnd["dlogits"][r] = g * (hot - p).abs() + (w * c).abs() * p * (ds + U * (3 * far + 8))
        bnd["dlogits"][r, a] += (w * c).abs() * (p[a] * el + 4 * U * (1 - p[a]))
    return {x: (val[x], bnd[x]) for x in val}
