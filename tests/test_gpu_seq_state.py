"""The recurrence's state in place (hT = h0, dh0 = dhT) with an odd number of channels in pairs: many more workgroups
than run at a time, so that some end before others begin, give the bits of a state kept apart."""
import pytest
import torch

from tests import seq_ref as R

pytestmark = pytest.mark.gpu

# 128 k + 1 channels, and other odd numbers; one, four and eight waves a tile, several tiles; forward alone in pairs
# (the last two)
SHAPES = [(4096, 1, 129), (20000, 1, 129), (2500, 1, 257), (3000, 20, 129), (700, 100, 257), (300, 150, 129),
          (2000, 5, 131), (64, 1, 129), (2, 300, 257)]


@pytest.mark.parametrize("B,T,D", SHAPES)
def test_state_in_place(B, T, D):
    from paper_2103_08802_amd import seq
    g = torch.Generator(device="cuda").manual_seed(B + T + D)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, gate, dh = (rnd(B, T, D).bfloat16() for _ in range(3))
    h, dx, dg = (torch.empty_like(x) for _ in range(3))
    h0, dhT = rnd(B, D), rnd(B, D)
    d = seq.scan_desc(x, gate, h, dh, dx, dg)
    n, w = seq.pnn_scan_sizes(d)
    states, ws = torch.empty(n // 4, device="cuda"), torch.empty(w + 256, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream

    def go(first, last, dlast, dfirst):
        seq.pnn_scan_fwd(d, x, gate, None, first, h, last, states, ws, s)
        seq.pnn_scan_bwd(d, x, gate, None, states, dh, dlast, dx, dg, dfirst, ws, s)
        return [t.clone() for t in (h, states, dx, dg, last, dfirst)]

    apart = go(h0, torch.empty_like(h0), dhT, torch.empty_like(dhT))
    keep = min(B, 40)
    ref = R.scan(x[:keep], gate[:keep], None, h0[:keep], dh[:keep], dhT[:keep])
    for name, t, ty in (("h", apart[0], "bf16"), ("hT", apart[4], "f32"), ("dx", apart[2], "bf16"),
                        ("dgate", apart[3], "bf16"), ("dh0", apart[5], "f32")):
        R.within(t[:keep], *ref[name], ty)
    a, b = h0.clone(), dhT.clone()
    for got, want in zip(go(a, a, b, b), apart):
        assert torch.equal(got, want)
