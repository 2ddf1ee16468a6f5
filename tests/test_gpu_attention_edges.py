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


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("part", ["all numbers", "some numbers"])
@pytest.mark.parametrize("name", ["band", "sparse", "half", "ragged batch", "tokens behind a prefix", "one row", "cut rows"])
def test_values_that_are_not_numbers_leave_lse_and_dv_right(name, part, dt):
    """lse does not depend on V, and dV = p^T dO not on V either: a V of NaN (its K is a number) spoils O and the gradients that the formula
    takes from it, and the other numbers of a head's O stay right where only some of V's are spoiled."""
    at = torch.cat([torch.ones(24, 3000, dtype=torch.bool), ragged([1] * 24, [40] * 24)], 1) if name == "cut rows" else PATTERNS[name]()
    p = problem(at, 2, 1, 64, dt)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    cols = at.any(0).nonzero().flatten()
    col = int(cols[len(cols) // 3])
    say("case", name, part, dt, "column", col)
    spoiled = torch.ones(64, dtype=torch.bool) if part == "all numbers" else torch.arange(64) % 5 == 0
    was = p.V[col].clone()
    p.V[col, :, spoiled] = float("nan")
    got = run(S, p)
    p.V[col] = was
    ref = reference(p)
    check({k: got[k] for k in ("lse", "dV")}, {k: ref[k] for k in ("lse", "dV")}, name)
    rows = at[:, col]
    nan = torch.isnan(got["O"].cpu())
    assert bool((nan == (rows[:, None, None] & spoiled)).all())
    check({"O": got["O"][:, :, (~spoiled).to(DEV)]}, {"O": tuple(t[:, :, ~spoiled] for t in ref["O"])}, name)
    clean, far = ~rows, ~at[rows].any(0)                 # rows without it, and the keys that none of the others has
    check({"dQ": got["dQ"][clean.to(DEV)], "dK": got["dK"][far.to(DEV)]},
          {"dQ": tuple(t[clean] for t in ref["dQ"]), "dK": tuple(t[far] for t in ref["dK"])}, name)
    assert bool(torch.isnan(got["dQ"][rows.to(DEV)]).all()) and bool(torch.isnan(got["dK"][at[rows].any(0).to(DEV)]).all())
