"""Norms around a block where the row's end cuts a 16-byte piece: every number of elements left over, in every layout of
rows over lanes, out of place against 64 bits and in place with the same bits."""
import pytest
import torch

from tests.test_gpu_norm import Case, _seq, _stream

pytestmark = pytest.mark.gpu

# the last whole piece's end: rows over 16 lanes (one piece a lane, two), 64, 256, 1024
BASES = {"bf16": [8, 120, 128, 248, 504, 1016, 2040, 4088, 5000, 8184], "f32": [4, 60, 64, 124, 252, 508, 1020, 2044, 2500, 4092]}


@pytest.mark.parametrize("dtype,base", [(d, b) for d in BASES for b in BASES[d]])
def test_every_rest_of_a_row(dtype, base):
    for rest in range(1, 8 if dtype == "bf16" else 4):
        for parts in ("pgrnwd", "prnw"):
            c = Case(19, 1, base + rest, dtype, parts, lead=rest % 3, pad=rest % 2)
            c.forward()
            c.check_forward()
            c.backward()
            c.check_backward(c.reference())


@pytest.mark.parametrize("dtype,width", [("bf16", 121), ("bf16", 515), ("bf16", 1029), ("bf16", 2053), ("bf16", 4099),
                                         ("f32", 259), ("f32", 1030), ("f32", 2049), ("f32", 4101)])
@pytest.mark.parametrize("parts", ["r", "gr", "pgrnwd"])
def test_in_place(dtype, width, parts):
    """h in the place of res, dres in that of dh: a lane's pieces are its own, also where it loads its neighbour's."""
    c = Case(300, 1, width, dtype, parts if "d" in parts else parts + "d")
    c.forward()
    c.backward()
    h, dres = c.h.clone(), c.dres.clone()
    c.backward(dres="dh")
    assert torch.equal(c.dh, dres)
    _seq().pnn_norm_fwd(c.desc, c.x, c.w1, c.gate, c.res, c.w2, c.res, c.y, _stream())
    assert torch.equal(c.res, h)
    c.intact()
