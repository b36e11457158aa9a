"""The sequence operators at sizes whose rules take other paths than small tensors': tables whose rows are cleared in
several launches and by their row bits, tensors larger than the caches, tiles of one workgroup after the other.  The
checks are those of tests/test_gpu_seq.py."""
import pytest
import torch

import tests.test_gpu_seq as T

pytestmark = pytest.mark.gpu

I32, I64 = torch.int32, torch.int64

EMBED = [
    # tokens' rows above 8 MB: the last launch clears by row bits what the sort's launches leave
    (4100, 520, 40003, "bf16", "bf16", I64, "mixed", 0, 0),      # split over the sort's launches, then 4128 rows by bits
    (4100, 521, 40003, "f32", "f32", I32, "mixed", 1, 3),        # the same with rows on odd elements
    (9000, 600, 3703, "bf16", "f32", I32, "mixed", 0, 8),        # every row by bits, the last word of them in part
    (9000, 600, 3703, "bf16", "bf16", I32, "none", 0, 0),        # ... none of which is set
    (2000, 1100, 5003, "f32", "bf16", I64, "mixed", 0, 0),       # sorted by one workgroup
    (20000, 120, 30011, "bf16", "bf16", I64, "plain", 0, 0),     # 32 rows to a clearing workgroup
    (140001, 16, 150001, "f32", "f32", I32, "mixed", 0, 0),      # histograms summed by a launch of their own
    # forward results above 32 MB; one run of all tokens
    (16400, 1030, 301, "bf16", "f32", I64, "mixed", 1, 1),
    (9000, 1000, 11, "f32", "f32", I32, "one", 0, 0),
]


@pytest.mark.parametrize("n,width,vocab,rows,table,tok,kind,lead,pad", EMBED)
def test_embed(n, width, vocab, rows, table, tok, kind, lead, pad):
    T.test_embed(n, width, vocab, rows, table, tok, kind, lead, pad)


SCAN = [
    (150, 600, 40, "bf16", "dense", "ragged", True, 0),          # sixteen waves, several tiles, not dealt
    (150, 600, 40, "f32", "halves", "ragged", True, 1),
    # above 32 MB
    (300, 40, 1401, "bf16", "halves", "ragged", True, 1),        # pairs
    (16, 600, 1801, "bf16", "dense", "ragged", True, 0),         # one channel a lane
    (4, 2100, 1000, "f32", "dense", "ragged", True, 0),          # dealt
    (1, 2100, 8100, "bf16", "dense", None, True, 0),             # dealt, forward in pairs
]


@pytest.mark.parametrize("B,T_,D,dtype,layout,lens,state,lead", SCAN)
def test_scan(B, T_, D, dtype, layout, lens, state, lead):
    T.test_scan(B, T_, D, dtype, layout, lens, state, lead)


DISTILL = [
    # gradients above 32 MB, with classes written again at their entries and labels
    (290, 60001, 64, "bf16", "bf16", 2.0, 0.5, True, True, 1, 0),
    (130, 65001, 300, "f32", "f32", 3.0, 0.5, True, True, 0, 3),
    (70, 140003, 50, "f32", "bf16", 4.0, 0.5, True, True, 0, 0),     # rows read twice
]


@pytest.mark.parametrize("n,V,k,dtype,td,tau,alpha,labelled,masked,lead,pad", DISTILL)
def test_distill(n, V, k, dtype, td, tau, alpha, labelled, masked, lead, pad):
    T.test_distill(n, V, k, dtype, td, tau, alpha, labelled, masked, lead, pad)
