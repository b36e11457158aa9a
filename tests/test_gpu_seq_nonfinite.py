"""The recurrence at the edges of its numbers: states and gradients that are not finite stay out of the steps behind a
sequence's end, and gates of plus and minus infinity hold or replace a state exactly, however large it is."""
import math

import pytest
import torch

from tests import seq_ref as R

pytestmark = pytest.mark.gpu

# one, four, eight and sixteen waves a tile; tiles dealt; pairs of channels; several tiles to a workgroup
SHAPES = [(3, 6, 5, "f32"), (4, 17, 96, "f32"), (3, 128, 40, "bf16"), (2, 300, 70, "f32"), (520, 300, 5, "f32"),
          (300, 40, 131, "bf16"), (150, 600, 40, "bf16")]


def _run(x, gate, lengths, h0, dh, dhT):
    from paper_2103_08802_amd import seq
    h, dx, dg = (torch.full_like(x, 77.0) for _ in range(3))
    hT, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    d = seq.scan_desc(x, gate, h, dh, dx, dg)
    n, w = seq.pnn_scan_sizes(d)
    states = torch.empty(n // 4, device="cuda")
    ws = torch.empty(w + 256, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    seq.pnn_scan_fwd(d, x, gate, lengths, h0, h, hT, states, ws, s)
    seq.pnn_scan_bwd(d, x, gate, lengths, states, dh, dhT, dx, dg, dh0, ws, s)
    return {"h": h, "hT": hT, "dx": dx, "dgate": dg, "dh0": dh0}


def _inputs(B, T, D, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x, gate, dh = (torch.randn(B, T, D, generator=g).to(R.DT[dtype]).cuda() for _ in range(3))
    lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
    lengths[0], lengths[1], lengths[-1] = T, T // 2, 0
    h0, dhT = (torch.randn(B, D, generator=g).cuda() for _ in range(2))
    return x, gate, dh, lengths.cuda(), h0, dhT


@pytest.mark.parametrize("what", ["x", "h0", "dhT", "dh"])
@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_steps_behind_the_end_stay_zero(B, T, D, dtype, what):
    """Channel 0 of every sequence meets an infinity or NaN; the steps behind the ends are zero all the same, and the
    other channels have the bits they have without."""
    x, gate, dh, lengths, h0, dhT = _inputs(B, T, D, dtype, B + T + D)
    want = _run(x, gate, lengths, h0, dh, dhT)
    bad = torch.tensor([math.inf, -math.inf, math.nan], device="cuda").repeat(B)[:B]
    t = {"x": x, "h0": h0, "dhT": dhT, "dh": dh}[what]
    if t.dim() == 2:
        t[:, 0] = bad
    else:
        t[:, 0, 0] = bad.to(t.dtype)
    got = _run(x, gate, lengths, h0, dh, dhT)
    behind = torch.arange(T, device="cuda") >= lengths[:, None]
    for name in ("h", "dx", "dgate"):
        assert not got[name][behind].any(), name            # NaN counts as true
    for name in got:
        assert torch.equal(got[name][..., 1:], want[name][..., 1:]), name


@pytest.mark.parametrize("B,T,D,dtype", SHAPES)
def test_infinite_gates_hold_and_replace(B, T, D, dtype):
    """f is 1 and 1 - f is 0 for a gate of +inf, the other way round for -inf: a state of 1e38 is gone after the one,
    an input of 1e38 never arrives with the other, and neither has a gradient from what it leaves out."""
    x, gate, dh, lengths, h0, dhT = _inputs(B, T, D, dtype, B + T + D + 1)
    g = torch.Generator().manual_seed(B * T)
    kind = torch.randint(0, 6, gate.shape, generator=g).cuda()
    kind[:, 0, 0], kind[:, 0, 1] = 0, 1
    gate[kind == 0], gate[kind == 1] = -math.inf, math.inf
    x[kind == 1] *= 1e37
    h0 *= 1e37
    dh *= 2.0 ** -7
    dhT *= 2.0 ** -7
    got = _run(x, gate, lengths, h0, dh, dhT)
    ref = R.scan(x, gate, lengths, h0, dh, dhT)
    for name in got:
        R.within(got[name], *ref[name], dtype if name in ("h", "dx", "dgate") else "f32")
