"""The norms' backward from the stored sum: refusals at the C ABI and of descriptions that do not say what they are given
(no GPU needed; refused calls enqueue nothing), and the gradients' reference against differences of its forward."""
import pytest
import torch

from tests import block_ref as R
from tests.test_block_abi import ALIGN, L, LARGE, NBWD, NULL, Q, SHAPE, S, P, _nb, _norm  # noqa: F401


def test_stored_sum_at_the_abi(L):  # noqa: F811
    assert _nb(L, _norm(stored=1), res=None) == NULL                     # a stored sum is needed
    assert _nb(L, _norm(stored=1), res=NBWD["res"] + 1) == ALIGN
    # it has h's strides, not the residual's
    far, back = Q.RowStride(1 << 60, 32), Q.RowStride(-96, 32)
    assert _nb(L, _norm(stored=1, h=far)) == LARGE and _nb(L, _norm(stored=1, h=back)) == SHAPE
    assert _nb(L, _norm(stored=1, res=back), dy=None) == NULL
    assert _nb(L, _norm(stored=0, res=back)) == SHAPE
    # x is looked at for its own norm and gate only
    d = _norm(post=0, stored=1, dx=Q.RowStride(90, 32))
    assert _nb(L, d, x=None, gate=None, dgate=None, dx=NBWD["dx"] + 1) == SHAPE
    d = _norm(post=0, stored=1)
    assert _nb(L, d, x=None, gate=None, dgate=None, dx=NBWD["dx"] + 1) == ALIGN
    assert _nb(L, _norm(stored=1), x=None) == NULL and _nb(L, d, x=None) == NULL
    assert _nb(L, _norm(post=0), x=None, gate=None, dgate=None) == NULL
    for o in ("dx", "dgate", "dres"):
        assert _nb(L, _norm(stored=1), **{o: NBWD["res"]}) == SHAPE
    # without a norm of the sum it is not looked at
    assert _nb(L, _norm(pre=0, stored=1), res=None, dy=None, dx=NBWD["dx"] + 1) == ALIGN


def _bwd(d, res):
    Q.pnn_norm_bwd(d, P, None, None, res, None, P + S, None, P + 2 * S + 1, None, None, None, None, False, None, None)


def test_descriptions_say_what_the_backward_is_given(L):  # noqa: F811
    x, res, h, y = (torch.zeros(4, 8) for _ in range(4))
    t = dict(res=res, h=h, y=y, dy=y, dx=y, pre=True)
    for place in (h, h.data_ptr(), h[:2]):
        with pytest.raises(ValueError, match="stored"):
            _bwd(Q.norm_desc(x, **t), place)
    with pytest.raises(ValueError, match="stored"):                      # described in place
        _bwd(Q.norm_desc(x, **{**t, "res": h}), h)
    # each of these gets as far as the pointer that is not aligned
    for d, given in ((Q.norm_desc(x, **t), res), (Q.norm_desc(x, **t), None), (Q.norm_desc(x, **t), P + 4 * S),
                     (Q.norm_desc(x, **t, stored=True), h), (Q.norm_desc(x, **t, stored=False), h),
                     (Q.norm_desc(x, **{**t, "res": h}, stored=True), h), (Q.norm_desc(x, **t, kept=True), h),
                     (Q.norm_desc(x, **t, kept=True), res)):
        with pytest.raises(Q.PnnError) as e:
            _bwd(d, given)
        assert e.value.status == ALIGN
    assert Q.norm_desc(x, **t, stored=True).stored == 1 and Q.norm_desc(x, **t).stored == 0
    d = Q.norm_desc(x, **t, kept=True)
    assert d.stored == 0 and Q._norm_sum(d, h) is res and Q._norm_sum(d, res) is res and Q._norm_sum(d, None) is None
    with pytest.raises(ValueError, match="kept"):
        _bwd(d, P + 4 * S)
    none = Q.norm_desc(x, **{**t, "res": None}, kept=True)
    assert Q._norm_sum(none, h) is None
    for bad in (dict(stored=True), dict(res=h), dict(h=None)):
        with pytest.raises(ValueError, match="kept"):
            Q.norm_desc(x, **{**t, **bad}, kept=True)
    # the place of a tensor that is gone says nothing
    gone = torch.zeros(4, 8)
    d, at = Q.norm_desc(x, **{**t, "h": gone}), gone.data_ptr()
    del gone
    with pytest.raises(Q.PnnError):
        _bwd(d, at)


@pytest.mark.parametrize("parts", ["p", "pg", "n", "rn", "prn", "pgrn"])
def test_reference_gradients_against_differences(parts):
    """In 64 bits: central differences of step e = 2^-17 leave (e^2 / 6) = 1e-11 times the third derivative along the way
    and the sums' roundings over e, at most some hundred 2^-53 of the summed magnitudes times 2^17: 2^-28 of them."""
    g = torch.Generator().manual_seed(len(parts))
    new = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    post, pre, shape, eps, alpha = "p" in parts, "n" in parts, (3, 2, 20), 1e-5, 0.75
    a = {"x": new(*shape), "w_post": 1 + 0.3 * new(20) if post else None, "gate": new(*shape) if "g" in parts else None,
         "res": new(*shape) if "r" in parts else None, "w_pre": 1 + 0.3 * new(20) if pre else None}
    dy, dh = new(*shape) if pre else None, new(*shape)

    def loss(**change):
        f = R.norm_fwd(*{**a, **change}.values(), post, pre, eps, alpha)
        t = [f["h"][0] * dh] + ([f["y"][0] * dy] if pre else [])
        return sum(x.sum() for x in t), sum(x.abs().sum() for x in t)

    got = R.norm_bwd(*a.values(), dy, dh, post, pre, eps, alpha)
    size = float(loss()[1])
    e = 2.0 ** -17
    for n, t in a.items():
        if t is None:
            continue
        way = new(*t.shape)
        name = {"res": "dres", "w_post": "dw_post", "w_pre": "dw_pre"}.get(n, "d" + n)
        want = float((got[name][0] * way).sum())
        two = [float(loss(**{n: t + s * e * way})[0]) for s in (1, -1)]
        assert abs((two[0] - two[1]) / (2 * e) - want) <= 2.0 ** -24 * size, (n, want)
