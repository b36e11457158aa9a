"""The largest class count that the distillation takes, 2^31 - 1: one row, with and without a term."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

V = (1 << 31) - 1
LEAD, MARK = 3, 77.0


def test_distill_of_the_most_classes():
    """Logits of zero: every class has 1 / V, so with a scale of 2^31 the gradient is 1 (to bf16) but for the label's
    class, 1 - 2^31 there.  Without a term it is zero.  Nothing is stored before or behind the row."""
    from paper_2103_08802_amd import seq
    z = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda")
    buf = torch.full((LEAD + V + 8,), MARK, dtype=torch.bfloat16, device="cuda")
    dz = buf[LEAD:LEAD + V].view(1, V)
    index = torch.full((1, 2), -1, dtype=torch.int32, device="cuda")
    teacher, loss = torch.zeros(1, 2, device="cuda"), torch.empty(1, device="cuda")
    labels = torch.tensor([-1], dtype=torch.int32, device="cuda")
    d = seq.distill_desc(z, teacher, dz, 1.0, 0.0, 2.0 ** 31)
    s = torch.cuda.current_stream().cuda_stream

    def frame():
        return bool((buf[:LEAD] == MARK).all()) and bool((buf[LEAD + V:] == MARK).all())

    seq.pnn_distill_fwd_bwd(d, z, index, teacher, labels, None, loss, dz, s)
    assert frame() and loss.item() == 0.0 and not dz.any()
    labels[0] = V - 1
    seq.pnn_distill_fwd_bwd(d, z, index, teacher, labels, None, loss, dz, s)
    assert frame() and abs(loss.item() - 31 * math.log(2)) < 1e-5
    assert bool((dz[0, :-1] == 1.0).all()) and dz[0, -1].item() == -2.0 ** 31
