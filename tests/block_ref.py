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
    # product and the split of the weighted values; the states': the split alone
    sums = 2 * U * (K + V + T + 64)
    way = sums + (BF * (1 + 2 ** -6) + 2 ** -16 if dtype == "bf16" else 0.0)
    held = sums + (2 ** -16 if dtype == "bf16" else 0.0)
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
                whole * S0.abs() + (A.abs() * until).t() @ X.abs(), held)
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
                whole * Z.abs() + abs(scale) * (Q.abs() * since).t() @ D.abs(), held)
            bnd["ds0"][b, h] += U * (we * whole * Z.abs() + abs(scale) * (Q.abs() * since * se).t() @ D.abs())
    return {x: (val[x], bnd[x]) for x in names}
