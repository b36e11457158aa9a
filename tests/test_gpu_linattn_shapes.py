"""Linear attention on the GPU against 64 bits in the shapes of its kernels (type, padded width, waves, rows shorter than
a piece, blocks of value columns, cut sequences) that the other tests do not reach; test_linattn_shapes.py checks on the
CPU that together they reach all.  And its states, which are sums of products kept to 24 bits."""
import pytest
import torch

from tests import block_ref as R
from tests.seq_ref import f64
from tests.test_gpu_linattn import Case

pytestmark = pytest.mark.gpu

SHAPES = [
    # B, T, H, kv, K, V, dtype, layout, ragged, state
    (16, 70, 8, 8, 128, 128, "bf16", "steps", True, True),        # four waves, two blocks, both directions
    (16, 45, 8, 4, 72, 100, "bf16", "heads", False, False),
    (16, 45, 8, 8, 72, 100, "f32", "steps", True, True),
    (16, 40, 8, 2, 100, 67, "bf16", "steps", False, True),        # a block that starts less than a piece before the end
    (16, 40, 8, 8, 200, 72, "bf16", "time", True, True),
    (16, 40, 8, 8, 200, 72, "f32", "steps", False, True),
    (4, 40, 12, 12, 200, 200, "bf16", "steps", True, True),
    (4, 40, 12, 6, 150, 194, "f32", "steps", False, True),
    (72, 33, 4, 2, 16, 100, "bf16", "steps", True, True),
    (72, 33, 4, 4, 60, 66, "f32", "steps", True, False),
    (1, 400, 2, 1, 200, 140, "bf16", "steps", False, True),       # cut, two blocks
    (2, 300, 1, 1, 130, 250, "f32", "heads", True, True),
    (1, 600, 2, 2, 128, 128, "bf16", "steps", False, True),       # cut, whole tiles
    (2, 300, 2, 1, 40, 135, "bf16", "steps", True, True),
    (2, 300, 2, 2, 40, 131, "f32", "steps", False, True),
    (1, 260, 1, 1, 90, 129, "f32", "steps", False, True),
    (1, 260, 1, 1, 100, 133, "bf16", "time", False, True),
    (2, 300, 2, 1, 200, 48, "bf16", "steps", True, True),
    (2, 300, 2, 1, 200, 48, "f32", "steps", True, True),
    (1, 300, 3, 3, 200, 100, "f32", "steps", False, True),
    (1, 300, 3, 3, 200, 100, "bf16", "steps", False, True),
    (2, 280, 2, 1, 56, 40, "bf16", "steps", True, True),
    (2, 280, 2, 1, 56, 40, "f32", "steps", True, True),
    (1, 260, 1, 1, 100, 60, "bf16", "steps", False, True),
    (3, 70, 2, 1, 5, 7, "bf16", "steps", True, True),             # rows shorter than a piece
    (2, 70, 2, 2, 2, 3, "f32", "heads", False, True),
    (1, 300, 2, 1, 3, 200, "bf16", "steps", False, True),
    (1, 300, 2, 2, 140, 1, "f32", "steps", False, True),
    (2, 50, 2, 1, 7, 200, "bf16", "time", True, True),
    (2, 50, 2, 1, 3, 200, "f32", "steps", True, True),
    (1, 300, 1, 1, 6, 9, "bf16", "steps", False, True),
    (1, 300, 1, 1, 1, 1, "f32", "steps", False, True),
    (40, 40, 10, 10, 100, 100, "bf16", "steps", True, True),      # more heads than four waves are for
    (40, 40, 10, 5, 100, 80, "f32", "steps", True, True),
    (20, 40, 20, 20, 40, 140, "bf16", "steps", True, True),
    (20, 40, 20, 20, 40, 140, "f32", "steps", False, True),
    (2, 64, 2, 1, 48, 100, "bf16", "steps", True, True),          # forwards of other widths than their backward's
    (2, 60, 2, 1, 100, 50, "bf16", "steps", False, True),
    (2, 60, 2, 2, 90, 180, "bf16", "heads", True, True),
    (2, 60, 2, 1, 180, 50, "bf16", "steps", True, False),
    (2, 60, 2, 1, 180, 100, "bf16", "steps", False, True),
    (1, 300, 2, 1, 64, 100, "f32", "steps", False, True),
    (2, 60, 2, 1, 100, 50, "f32", "steps", True, True),
    (2, 60, 2, 2, 100, 100, "f32", "time", False, True),
    (1, 300, 2, 2, 100, 100, "f32", "steps", False, True),
    (2, 60, 2, 2, 90, 180, "f32", "steps", True, True),
    (2, 60, 2, 1, 180, 100, "f32", "heads", False, True),
    (1, 300, 2, 2, 2, 200, "f32", "steps", False, True),
]


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c)))
def test_every_shape(case):
    c = Case(*case, lead=1, pad=1) if case[5] % 2 else Case(*case)
    c.forward()
    c.backward()
    c.check(c.reference())


@pytest.mark.parametrize("T,K,V", [(40, 128, 128), (300, 64, 96), (70, 200, 136)])
def test_states_are_sums_of_24_bit_terms(T, K, V):
    """bf16: a term of sT is k (lambda^n v), lambda^n v split into three bf16 parts: what is left of it is at most 2^-24 of
    it.  A power is off by (2 n |ln lambda| + 4) U, 6 U where lambda^n is 1 / e; a sum of about 8 such terms in an order of
    32 and over chunks by a few U of its terms.  Errors of independent terms add up as the terms themselves do, so the
    state is off by under 12 U of its norm, 7e-7.  Two parts would leave up to 2^-16 of every term, 2.7e-6 on average.
    ds0's terms, q (lambda^n scale do), likewise."""
    c = Case(2, T, 2, 2, K, V, "bf16")
    c.decay.fill_(-0.125)
    c.s0.zero_()
    c.dsT.zero_()
    c.forward()
    c.backward()
    ref = R.linattn(c.q, c.k, c.v, c.decay, None, c.s0, c.desc.scale, "bf16", c.dout, c.dsT)
    for n in ("sT", "ds0"):
        value = ref[n][0]
        assert float((f64(getattr(c, n)) - value).norm() / value.norm()) <= 12 * R.U, n
    assert torch.isfinite(c.sT).all()
