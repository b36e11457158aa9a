"""Outputs of linear attention, norms and the policy loss in the place of another tensor of the call: refused at the C ABI
unless the entry point says that they may stand there.  No GPU needed: refused calls enqueue nothing."""
import pytest

from tests.test_block_abi import (L, LBWD, LFWD, NBWD, NFWD, P, POL, Q, S, SHAPE, _lb, _lf, _lin, _nb, _nf, _norm, _pol,  # noqa: F401
                                  _policy)

HEADS = {n: Q.HeadStride(1 << 20, 1 << 10, 24) for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")}
FWD = dict(LFWD, lengths=P + 20 * S, s0=P + 21 * S, sT=P + 22 * S, ws=P + 23 * S)
BWD = dict(LBWD, lengths=P + 20 * S, s0=P + 21 * S, dsT=P + 22 * S, ds0=P + 23 * S, ws=P + 24 * S)


@pytest.mark.parametrize("out", ["o", "sT"])
def test_linattn_forward(L, out):  # noqa: F811
    d = _lin(length=1000, kv_heads=4, **HEADS)              # cut: a workspace is used
    for k in FWD:
        if k != out and {k, out} != {"s0", "sT"}:
            assert _lf(L, d, **{**FWD, out: FWD[k]}) == SHAPE, k


@pytest.mark.parametrize("out", ["dq", "dk", "dv", "ds0"])
def test_linattn_backward(L, out):  # noqa: F811
    for k in BWD:
        if k != out:
            assert _lb(L, _lin(), **{**BWD, out: BWD[k]}) == SHAPE, k


def test_linattn_without_steps(L):  # noqa: F811
    """No steps: q, k, v, o have no elements, the states have."""
    assert _lf(L, _lin(length=0), **{**FWD, "sT": FWD["log_decay"]}) == SHAPE
    assert _lb(L, _lin(length=0), **{**BWD, "ds0": BWD["s0"]}) == SHAPE


@pytest.mark.parametrize("out", ["h", "y"])
def test_norm_forward(L, out):  # noqa: F811
    t = dict(NFWD, w_pre=P + 128)
    for k in t:
        if k != out and (out, k) != ("h", "res"):
            assert _nf(L, _norm(), **{**t, out: t[k]}) == SHAPE, k


@pytest.mark.parametrize("out", ["dx", "dgate", "dres", "dw_post", "dw_pre"])
def test_norm_backward(L, out):  # noqa: F811
    t = dict(NBWD, w_pre=P + 128, ws=P + 20 * S)
    for stored in (0, 1):
        for k in t:
            if k not in (out, "accumulate") and (out, k) != ("dres", "dh"):
                assert _nb(L, _norm(stored=stored), **{**t, out: t[k]}) == SHAPE, k


@pytest.mark.parametrize("out", ["loss", "logp", "dz"])
def test_policy(L, out):  # noqa: F811
    for k in POL:
        if k != out and (out, k) != ("dz", "z"):
            assert _pol(L, _policy(), **{out: POL[k]}) == SHAPE, k
