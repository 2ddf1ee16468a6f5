"""Attention over a stored pattern where its inputs are at an edge: nothing at all, biases that leave no room for a row's logarithm in
32 bits, values that are not numbers, the default allocator, calls beyond a launch.  Bounds as in tests/attention_util.py."""
import pytest
import torch

import paper_2202_04305_amd as sp
from attention_util import reference
from gpu_util import say, DEV
from test_gpu_attention import BF16, F16, F32, PATTERNS, band, check, code, pack, problem, ragged, run

pytestmark = pytest.mark.gpu


@pytest.fixture
def poisoned(monkeypatch):
    """Fresh memory that holds NaN (bytes of 255 in a workspace), so that nothing counts on zeros."""
    empty = torch.empty

    def filled(*a, **k):
        t = empty(*a, **k)
        return t.fill_(float("nan") if t.is_floating_point() else 255 if t.dtype == torch.uint8 else 0)
    monkeypatch.setattr(torch, "empty", filled)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("m,n", [(0, 5), (5, 0), (0, 0), (5, 7)])
def test_gradients_without_pairs_are_zeros(m, n, dt, poisoned):
    """The bias's among them, also where there is not one row: a workspace of no bytes has no address."""
    for buckets in (0, 8):
        p = problem(torch.zeros(m, n, dtype=torch.bool), 2, 1, 16, dt, buckets=buckets, positions=(torch.arange(m), torch.arange(n)), max_distance=20)
        S = sp.sp_prepare_attention(pack(p.at), grad=True)
        got = run(S, p)
        torch.cuda.synchronize()
        assert not got["O"].any() and bool((got["lse"] == float("-inf")).all())
        for k in ("dQ", "dK", "dV") + (("dT",) if buckets else ()):
            assert got[k].shape == {"dQ": (m, 2, 16), "dK": (n, 1, 16), "dV": (n, 1, 16), "dT": (8, 2)}[k]
            assert not got[k].any(), (k, got[k])
