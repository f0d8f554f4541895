"""Kernels whose dynamic shared memory comes to just the 48 KB that need no permission: their static arrays count too."""
import pytest
import torch

import paper_2604_08971_b200 as sentry
import synth
from tests import parity
from tests.parity import TOL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sn():
    s = sentry.Sentry(0)
    yield s
    s.close()


# (four bytes a unit)
@pytest.mark.parametrize("n", [8193, 11900, 11999, 12288, 12289])
def test_gate_select_long_rows(sn, n):
    S, k = 8, n // 3
    scores = torch.randn((S, n), generator=torch.Generator().manual_seed(n))
    masks = torch.tensor([7, 0, 3], dtype=torch.int32)
    want = torch.sort(torch.sort(scores, dim=1, descending=True, stable=True).indices[:, :k], dim=1).values[masks.long()]
    gs, gm = scores.cuda(), masks.cuda()
    assert torch.equal(sn.gate_select(gs, gm, k).cpu().long(), want) and sn.last_status() == 0
    (multi,) = sn.gate_select_multi([(gs, gm, k, 0)])
    assert torch.equal(multi.cpu().long(), want)
    if n <= 12288:                                  # what the allocation-free entry point takes
        kept, status = torch.empty((3, k), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        sentry.gate_select_static(gs, gm, k, kept, status=status)
        assert torch.equal(kept.cpu().long(), want) and status.item() == 0


# (selection: six bytes a token, attention three, scores two)
@pytest.mark.parametrize("T", [7990, 8192, 16384, 24576])
def test_plain_alu_attention_of_long_sequences(sn, T):
    w = synth.Workload("window_T%d" % T, "f32", 1, (T // 2, T - T // 2), 16, 2, 1, 16, 16, 1, 8, "all", 1)
    inp = synth.generate(w, lambda tv: sentry.num_active_queries(tv, w.c))
    kept_h, _ = parity.gate_lists(sn, inp)
    assert parity.attend_parity(sn, inp, kept_h)[0] <= TOL[w.dtype]
