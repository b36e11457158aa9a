"""Scalars of the sequence operators at the ends of their ranges: taken or refused (no GPU needed)."""
import os

import pytest

B = pytest.importorskip("paper_2103_08802_amd.binding")
from paper_2103_08802_amd import seq as Q  # noqa: E402

VALUE = -10


@pytest.mark.parametrize("tau,status", [(3.5e-39, VALUE), (4.2e-39, VALUE), (4.3e-39, 0), (1e-30, 0), (1e19, 0), (3e19, VALUE)])
def test_distill_temperature(tau, status):
    """log2(e) / tau has to be finite (below tau = 4.2e-39 every logit's exponent was infinity times a difference), and
    so has alpha tau^2; a call without rows says which descriptions are taken."""
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libpnn.so not built")
    d = Q.DistillDesc(dtype=0, teacher_dtype=0, rows=0, classes=4, top=2, logit_stride=4, grad_stride=4, top_stride=2,
                      temperature=tau, alpha=1.0, scale=1.0)
    assert Q.lib().pnn_distill_fwd_bwd(d, None, None, None, None, None, None, None, None) == status
