"""Attention over a stored pattern where its inputs are at an edge: nothing at all, biases that leave no room for a row's logarithm in
32 bits, values that are not numbers, the default allocator, calls beyond a launch.  Bounds as in tests/attention_util.py."""
import pytest
import torch

import paper_2202_04305_amd as sp
from attention_util import reference
from gpu_util import say, DEV
from test_gpu_attention import BF16, F16, F32, PATTERNS, band, check, code, pack, problem, ragged, random_pattern, run

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


LOWEST = [(F16, -2048.0), (F16, -65504.0), (F32, -65504.0), (BF16, -65504.0), (BF16, -1e7), (F32, -1e8), (F32, -1e9), (BF16, -1e9), (F32, torch.finfo(F32).min),
          (BF16, torch.finfo(BF16).min)]


def far_below(at, H, Hk, D, dt, low, rows, seed=0):
    """A problem whose bucket 0 holds `low`, of which `rows` have nothing else, and what has to come out of it.  All scores are the bias
    alone (Q and K have no number in common that is not zero), so they are exact in 32 bits, and what a row of equal scores weighs does not
    depend on them: those rows are taken with a bias of 0, the others without the pairs of bucket 0, whose weight e^low is 0."""
    m, n = at.shape
    kpos = torch.tensor([10, 8, 6, 2])[torch.arange(n) % 4]
    qpos = torch.full((m,), 9)                           # distances of 1, -1, -3, -7: buckets 0 to 3
    qpos[rows] = 1                                       # every key ahead: bucket 0
    p = problem(at, H, Hk, D, dt, seed=seed, buckets=4, positions=(qpos, kpos), max_distance=8, bidirectional=False)
    p.Q[:, :, D // 2:] = 0
    p.K[:, :, :D // 2] = 0
    p.bias[0] = low
    ahead = (p.kpos[None, :] >= p.qpos[:, None])
    whole = ~(at & ~ahead).any(1)                        # `rows`, and those of a few entries that all lie ahead
    lowest, table = p.bias[0].clone(), p.bias
    p.at, p.bias = at & whole[:, None], torch.zeros_like(table)
    equal = reference(p)
    p.at, p.bias = at & ~whole[:, None] & ~ahead, table
    rest = reference(p)
    p.at = at
    ref = {k: tuple(a + b for a, b in zip(equal[k], rest[k])) for k in ("O", "dQ", "dK", "dV", "dT")}
    lse, tol = (torch.where(whole[None, :], a, b) for a, b in zip(equal["lse"], rest["lse"]))
    some = whole & at.any(1)
    assert bool(some[rows].any())
    lse[:, some] += lowest.double()[:, None]
    tol[:, some] += 2.0 ** -24 * abs(low)
    ref["lse"] = lse, tol
    for k in ("O", "dQ", "dK", "dV"):                    # the bounds say something
        assert float(ref[k][1].max()) <= 0.3 * float(ref[k][0].abs().max()), k
    return p, ref


@pytest.mark.parametrize("dt,low", LOWEST)
@pytest.mark.parametrize("name", ["dense", "one row", "sparse", "tokens behind a prefix", "cut rows", "all rows"])
@pytest.mark.parametrize("heads", [(2, 1), (6, 1), (40, 2)])
def test_rows_of_nothing_but_the_lowest_bias_weigh_their_keys_alike(heads, name, dt, low):
    """lse = low + log n is low in 32 bits, so weights e^(s - lse) are all 1 where they should be 1 / n."""
    at = torch.ones(20, 3000, dtype=torch.bool) if name == "cut rows" else PATTERNS["dense" if name == "all rows" else name]()
    rows = slice(None) if name in ("all rows", "one row") else [3, 4, 11]
    p, ref = far_below(at, heads[0], heads[1], 32, dt, low, rows)
    say("case", name, heads, dt, low)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    check(run(S, p), ref, "%s %s" % (name, low))


@pytest.mark.parametrize("dt", [BF16, F32])
def test_rows_far_below_zero_from_a_recorded_graph(dt):
    at = torch.ones(70, 900, dtype=torch.bool)
    p, ref = far_below(at, 4, 2, 64, dt, float(torch.finfo(dt).min), [0, 33, 69])
    S = sp.sp_prepare_attention(pack(at), grad=True)
    o = p.options(DEV)
    Q, K, V, dO = (t.to(DEV) for t in (p.Q, p.K, p.V, p.dO))
    eager = run(S, p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, lse = sp.sp_attention(S, Q, K, V, **o)
        grads = sp.sp_attention_grad(S, Q, K, V, O, lse, dO, **o)
    for rep in range(3):
        for t in (O, lse) + grads:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = dict(zip(("O", "lse", "dQ", "dK", "dV", "dT"), (O, lse) + grads))
        check(got, ref, "replay %d" % rep)
        for k, t in got.items():
            assert torch.equal(t, eager[k]), k


@pytest.mark.parametrize("low", [-3e3, -1e6, -1e7, -1e8, -1e9, 1e6, 1e8])
@pytest.mark.parametrize("name", ["dense", "sparse", "tokens behind a prefix", "cut rows"])
def test_weights_sum_to_one_where_scores_have_wide_steps(name, low):
    """Products of any size beside a bias that leaves them few bits: which weights come out depends on how scores round, but each row's sum
    to 1, so the rows of dV add up to those of dO.  A weight's exponent is at most 64 where it counts (2^-64 of the sum), rounded to 64 * 2^-24 of
    the weight, once where the sum is made and once where the weight is; sums of n terms add n * 2^-24."""
    at = torch.ones(20, 3000, dtype=torch.bool) if name == "cut rows" else PATTERNS[name]()
    m, n = at.shape
    p = problem(at, 2, 1, 32, F32, buckets=4, positions=(torch.arange(m), torch.arange(n)), max_distance=8, bidirectional=False)
    p.Q, p.K = p.Q * 4, p.K * 4
    p.bias[:] = low
    say("case", name, low)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got = run(S, p)
    there = at.any(1)
    want, most = p.dO[there].double().sum((0, 1)), p.dO[there].double().abs().sum((0, 1))
    tol = (2 * 64 + 2 * max(m, n) + 16) * 2.0 ** -24 * most
    x = got["dV"].double().cpu().sum((0, 1))
    assert bool(((x - want).abs() <= tol).all()), float(((x - want).abs() / tol).max())
    assert bool(torch.isfinite(got["dQ"]).all()) and bool(torch.isfinite(got["dK"]).all())


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("name", ["dense", "sparse", "one row", "tokens behind a prefix"])
def test_a_row_that_is_not_a_number_spoils_the_biases_of_its_own_distances_only(name, dt):
    """dTable[b] sums over the pairs of bucket b: a row whose dO is NaN reaches the buckets that its pairs have."""
    at = PATTERNS[name]()
    m, n = at.shape
    qpos, kpos = torch.arange(m) % 50, torch.arange(n) % 50
    row = m // 2
    qpos[row] = 2000                                     # all of its keys lie far behind: one bucket, the last of that side
    p = problem(at, 2, 1, 32, dt, buckets=16, positions=(qpos, kpos), max_distance=100)
    p.dO[row] = 0
    ref = reference(p)
    p.dO[row] = float("nan")
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got = run(S, p)
    others = torch.arange(16) != 7
    check({"dT": got["dT"][others.to(DEV)]}, {"dT": tuple(t[others] for t in ref["dT"])}, name)
    if at[row].any():
        assert bool(torch.isnan(got["dT"][7]).all())


class _DefaultAllocator:
    """No callbacks: the library's own allocator."""
    alloc_cb, free_cb = sp.binding._ALLOC_FN(), sp.binding._FREE_FN()


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("m,n,pairs", [(20, 30, 0), (1000, 30, 0), (0, 4, 0), (4, 0, 0), (0, 0, 0), (200, 100, 500), (1, 1, 1)])
def test_default_allocator(m, n, pairs, grad):
    """Nothing stored needs no chunks, and an allocator that is asked for no bytes gives no address."""
    at = torch.zeros(m, n, dtype=torch.bool)
    g = torch.Generator().manual_seed(6)
    if pairs:
        at[torch.randint(m, (pairs,), generator=g), torch.randint(n, (pairs,), generator=g)] = True
    rows, cols = (t.to(DEV).contiguous() for t in at.nonzero(as_tuple=True))
    S = sp.sp_pack(sp.sp_encode((0, 1), None, 32, 32), (m, n), [rows, cols], torch.zeros(rows.numel(), device=DEV), allocator=_DefaultAllocator())
    sp.sp_prepare_attention(S, grad=grad)
    p = problem(at, 2, 1, 16, F32)
    check(run(S, p, grad), reference(p, grad))
    torch.cuda.synchronize()
    S.free()


def test_calls_of_more_workgroups_than_a_launch_has_are_refused():
    """A launch has fewer than 2^32 threads in a direction: 2^24 workgroups of 256.  2^24 rows in blocks of 128, 128 heads."""
    m = 1 << 24
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    S = sp.sp_pack(sp.sp_encode((0, 1), None, 32, 32), (m, 8), [none, none], torch.zeros(0, device=DEV))
    sp.sp_prepare_attention(S, grad=True)
    row = torch.zeros(1, 128, 1, dtype=BF16, device=DEV)
    Q, K = row.expand(m, -1, -1), torch.zeros(8, 128, 1, dtype=BF16, device=DEV)
    O = torch.empty(m, 128, 1, dtype=BF16, device=DEV)
    lse = torch.empty(128, m, device=DEV)
    assert code(sp.sp_attention, S, Q, K, K, O=O, lse=lse) == 11
    assert code(sp.sp_attention_grad, S, Q, K, K, O, lse, O, dQ=O, dK=K, dV=K) == 11


def test_more_blocks_of_rows_than_a_launch_has_workgroups():
    """2^29 rows and a few, of which three store anything: the inspector looks at 2^24 blocks of 32."""
    m, H = (1 << 29) + 5, 1
    rows, cols = torch.tensor([7, 7, (1 << 28) + 1, m - 1, m - 1, m - 1]), torch.tensor([1, 5, 0, 0, 3, 7])
    S = sp.sp_pack(sp.sp_encode((0, 1), None, 32, 32), (m, 8), [rows.to(DEV), cols.to(DEV)], torch.zeros(6, device=DEV))
    sp.sp_prepare_attention(S)
    some = torch.unique(rows)
    at = torch.zeros(3, 8, dtype=torch.bool)
    at[torch.searchsorted(some, rows), cols] = True
    p = problem(at, H, 1, 4, BF16, train=False)
    Q = torch.zeros(m, 1, 4, dtype=BF16, device=DEV)
    Q[some.to(DEV)] = p.Q.to(DEV)
    O, lse = sp.sp_attention(S, Q, p.K.to(DEV), p.V.to(DEV))
    check({"O": O[some.to(DEV)], "lse": lse[:, some.to(DEV)]}, reference(p, False))
    assert int((lse != float("-inf")).sum()) == 3 and int((O != 0).any(2).sum()) == 3


def by_abi(S, p, grads=True, **without):
    """The calls of the C ABI with pointers that may be NULL left out."""
    from paper_2202_04305_amd import binding
    import ctypes
    L, st = sp.load_library(), torch.cuda.current_stream().cuda_stream
    o = p.options(DEV)
    Q, K, V, dO = (t.to(DEV) for t in (p.Q, p.K, p.V, p.dO))
    a = binding._attention_problem(S, Q, K, V, o["scale"], o.get("causal", False), o.get("qpos"), o.get("kpos"), o.get("bias"), o.get("max_distance", 128),
                                   o.get("bidirectional", True))
    keep = [o, Q, K, V, dO]

    def work(grad):
        size = ctypes.c_size_t()
        assert L.sp_attention_workspace(S._h, ctypes.byref(a), grad, ctypes.byref(size)) == 0
        keep.append(torch.full((max(size.value, 1),), 255, dtype=torch.uint8, device=DEV))
        return keep[-1].data_ptr(), size.value
    out = {"O": torch.empty_like(Q), "lse": torch.empty(Q.shape[1], Q.shape[0], device=DEV)}
    lse = None if "lse" in without else out["lse"].data_ptr()
    assert L.sp_attention(S._h, ctypes.byref(a), out["O"].data_ptr(), out["O"].stride(0), out["O"].stride(1), lse, *work(0), st) == 0
    if lse is None:
        torch.cuda.synchronize()
        return {"O": out["O"]}
    g = binding.SpAttentionGrads()
    for k, like in (("dQ", Q), ("dK", K), ("dV", V)):
        out[k] = torch.empty_like(like)
    for k, ld, hd, t in (("O", "ldo", "hdo", out["O"]), ("dO", "lddo", "hddo", dO), ("dQ", "lddq", "hddq", out["dQ"]), ("dK", "lddk", "hddk", out["dK"]), ("dV", "lddv", "hddv", out["dV"])):
        setattr(g, k, t.data_ptr()); setattr(g, ld, t.stride(0)); setattr(g, hd, t.stride(1))
    g.lse = lse
    assert L.sp_attention_grad(S._h, ctypes.byref(a), ctypes.byref(g), *work(1), st) == 0
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("name", ["band", "sparse", "tokens behind a prefix", "one row"])
def test_outputs_that_may_be_left_out(name, dt):
    """lse NULL, and dTable NULL with a bias: the other outputs are the same bits."""
    at = PATTERNS[name]()
    p = problem(at, 4, 2, 32, dt, buckets=16, positions=(torch.arange(at.shape[0]), torch.arange(at.shape[1])), max_distance=60)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    want, ref = run(S, p), reference(p)
    assert torch.equal(by_abi(S, p, lse=None)["O"], want["O"])
    got = by_abi(S, p)                                   # rows may be cut otherwise than with the table's gradient
    del ref["dT"]
    check(got, ref, name)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("D", [8, 32, 40, 64, 96, 128, 160, 256])
def test_the_largest_tables_fit_beside_every_head_size(D, dt):
    """64 buckets over distances of up to 4096, in every way of making tiles: the tables and the sums by bucket share the LDS with the rows."""
    if dt == F32 and D > 128:
        pytest.skip("refused: does not fit a lane's registers")
    say("case", D, dt)
    g = torch.Generator().manual_seed(D)
    few, many = torch.rand(20, 700, generator=g) < 0.8, ragged([130, 33], [165, 100])
    for at, heads in ((few, (2, 1)), (few, (6, 1)), (torch.ones(1, 300, dtype=torch.bool), (40, 1)), (many, (2, 1))):
        m, n = at.shape
        where = torch.randint(-4500, 4500, (m,), generator=g), torch.randint(-4500, 4500, (n,), generator=g)
        p = problem(at, heads[0], heads[1], D, dt, buckets=64, positions=where, max_distance=4096, bidirectional=D % 16 == 0)
        S = sp.sp_prepare_attention(pack(at), grad=True)
        check(run(S, p), reference(p), "D %d heads %s" % (D, heads))


@pytest.mark.parametrize("made", ["sp_convert", "sp_add", "sp_spgemm"])
def test_patterns_that_other_calls_have_made(made):
    a, b = random_pattern(90, 70, 0.1, 1), random_pattern(90, 70, 0.1, 2)
    enc = sp.sp_encode((0, 1), (0, 1), 32, 32)

    def ones(at, order=(0, 1)):
        rows, cols = (t.to(DEV).contiguous() for t in at.nonzero(as_tuple=True))
        return sp.sp_pack(sp.sp_encode((0, 1), order, 32, 32), at.shape, [rows, cols], torch.ones(rows.numel(), device=DEV))
    if made == "sp_convert":
        at, S = a, sp.sp_convert(ones(a, (1, 0)), enc)
    elif made == "sp_add":
        at, S = a | b, sp.sp_add(ones(a), ones(b), enc)
    else:
        at, S = (a.float() @ b.t().float()) > 0, sp.sp_spgemm(ones(a), ones(b.t().contiguous()), enc)
    p = problem(at, 4, 2, 32, BF16)
    sp.sp_prepare_attention(S, grad=True)
    check(run(S, p), reference(p), made)
    assert sp.sp_tensor_info(S).derivedBytes > 0


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("name", ["one row", "band", "sparse", "half", "ragged batch", "tokens behind a prefix", "empty rows"])
def test_causal_by_positions_in_no_order(name, dt):
    at = PATTERNS[name]()
    g = torch.Generator().manual_seed(11)
    for heads, buckets in (((2, 2), 0), ((6, 1), 0), ((2, 1), 16), ((6, 1), 16)):
        where = torch.randint(-60, 60, (at.shape[0],), generator=g), torch.randint(-60, 60, (at.shape[1],), generator=g)
        p = problem(at, heads[0], heads[1], 40, dt, buckets=buckets, positions=where, causal=True, max_distance=50, bidirectional=heads[1] == 2)
        S = sp.sp_prepare_attention(pack(at), grad=True)
        check(run(S, p), reference(p), "%s %s %d" % (name, heads, buckets))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("name", ["dense", "sparse", "one row", "tokens behind a prefix"])
def test_a_bias_that_is_not_a_number_reaches_the_rows_that_have_its_distances_only(name, dt, bad):
    at = PATTERNS[name]()
    m, n = at.shape
    p = problem(at, 4, 2, 32, dt, buckets=16, positions=(torch.arange(m) % 37, torch.arange(n) % 41), max_distance=100)
    if m > 1:
        p.qpos[m // 2] = 2000                            # all of this row's keys in bucket 7, which no other row has
    else:
        p.bias[7] = 0
    p.bias[7] = bad
    rows = torch.arange(m) != (m // 2 if m > 1 else -1)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    p.dO[~rows] = 0
    got = run(S, p)
    p.bias[7], p.at = 0, at & rows[:, None]
    ref = reference(p)
    keys = ~at[~rows].any(0)
    check({"O": got["O"][rows.to(DEV)], "lse": got["lse"][:, rows.to(DEV)], "dQ": got["dQ"][rows.to(DEV)], "dK": got["dK"][keys.to(DEV)], "dV": got["dV"][keys.to(DEV)]},
          {"O": tuple(t[rows] for t in ref["O"]), "lse": tuple(t[:, rows] for t in ref["lse"]), "dQ": tuple(t[rows] for t in ref["dQ"]),
           "dK": tuple(t[keys] for t in ref["dK"]), "dV": tuple(t[keys] for t in ref["dV"])}, name)
    others = torch.arange(16) != 7
    check({"dT": got["dT"][others.to(DEV)]}, {"dT": tuple(t[others] for t in ref["dT"])}, name)
    if m > 1 and at[m // 2].any():
        assert bool(torch.isnan(got["O"][m // 2]).all())


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("name", ["band", "sparse", "tokens behind a prefix", "cut rows"])
def test_infinite_values_and_gradients_stay_with_their_rows(name, dt):
    """A value of infinity, and a dO of infinity in another row."""
    at = torch.cat([torch.ones(24, 3000, dtype=torch.bool), ragged([1] * 24, [40] * 24)], 1) if name == "cut rows" else PATTERNS[name]()
    p = problem(at, 2, 1, 32, dt)
    col = at.shape[1] - 1 if name != "sparse" and name != "band" else int((at.sum(0) + 1000 * (at.sum(0) == 0)).argmin())
    row = int((~at[:, col]).nonzero()[0])
    was = p.V[col].clone(), p.dO[row].clone()
    p.V[col], p.dO[row] = float("inf"), float("-inf")
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got = run(S, p)
    p.V[col], p.dO[row] = was
    ref = reference(p)
    has = at[:, col]
    check({"O": got["O"][(~has).to(DEV)], "lse": got["lse"]}, {"O": tuple(t[~has] for t in ref["O"]), "lse": ref["lse"]}, name)
    assert not bool(torch.isfinite(got["O"][has.to(DEV)]).any())
    rows, keys = ~has, ~at[row] & ~at[has].any(0)
    rows[row] = False
    check({"dQ": got["dQ"][rows.to(DEV)], "dK": got["dK"][keys.to(DEV)], "dV": got["dV"][(~at[row]).to(DEV)]},
          {"dQ": tuple(t[rows] for t in ref["dQ"]), "dK": tuple(t[keys] for t in ref["dK"]), "dV": tuple(t[~at[row]] for t in ref["dV"])}, name)


@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("heads", [(4, 4), (6, 1), (40, 1)])
@pytest.mark.parametrize("kind", ["sequences", "with a bias", "narrow band", "single rows"])
def test_dq_of_short_rows_has_two_roundings(kind, heads, dt):
    """ds and dQ are rounded to 16 bits, each by a like error in the mean square, so dQ's is sqrt(2) times that of one rounding.  D made of an O of 16
    bits adds one that is as large as ds' own for rows of few columns: it has to be made good.  (The spread of a mean square over 20,000
    numbers is below 1 %; 1.5 leaves 6 %.)"""
    at = band(600, 600, 12) if kind == "narrow band" else ragged([1] * 150, [20] * 150) if kind == "single rows" else ragged([25, 17, 31] * 8, [25, 17, 31] * 8)
    m, n = at.shape
    more = dict(buckets=32, positions=(torch.arange(m), torch.arange(n)), max_distance=128) if kind in ("with a bias", "narrow band") else {}
    p = problem(at, heads[0], heads[1], 64, dt, seed=3, **more)
    say("case", kind, heads, dt)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got, ref = run(S, p), reference(p)
    for k in ("dQ", "dK"):
        want = ref[k][0]
        error, one = (got[k].double().cpu() - want).norm(), (want.to(dt).double() - want).norm()
        say(k, float(error / one))
        assert float(error) <= 1.5 * float(one), (k, float(error / one))
    check(got, ref, kind)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("name", ["dense", "sparse", "one row", "tokens behind a prefix"])
def test_a_score_of_infinity_makes_its_row_nan_and_no_other(name, dt):
    at = PATTERNS[name]()
    p = problem(at, 2, 1, 32, dt, train=False)
    col = int((at.sum(0) + 1000 * (at.sum(0) == 0)).argmin())
    p.Q[:, :, 0] = p.Q[:, :, 0].abs() + 4
    p.K[col] = 0
    p.K[col, :, 0] = 3e38
    p.scale = 1.0
    S = sp.sp_prepare_attention(pack(at))
    got = run(S, p, False)
    p.K[col] = 0
    ref, rows = reference(p, False), ~at[:, col]
    check({"O": got["O"][rows.to(DEV)], "lse": got["lse"][:, rows.to(DEV)]}, {"O": tuple(t[rows] for t in ref["O"]), "lse": tuple(t[:, rows] for t in ref["lse"])}, name)
    assert bool(torch.isnan(got["O"][(~rows).to(DEV)]).all()) and bool(torch.isnan(got["lse"][:, (~rows).to(DEV)]).all())


@pytest.mark.parametrize("buckets", [0, 8])
def test_gradients_at_offsets_beyond_32_bits(buckets):
    """Keys' rows more than 2^31 numbers behind the first, queries' rows 2^30 numbers apart, gradients among them; nothing else is written."""
    n, ld, D, m = 150_000, 16_384, 32, 5
    at = torch.zeros(m, n, dtype=torch.bool)
    g = torch.Generator().manual_seed(9)
    at[:, torch.randint(n, (60,), generator=g)] = True
    at[:3, n - 40:] = True
    at[3] = False
    p = problem(at, 2, 1, D, BF16, buckets=buckets, positions=(torch.arange(m) * 30_000, torch.arange(n)), max_distance=2000)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    wide = torch.empty(n * ld, dtype=BF16, device=DEV).view(n, ld)
    K, V, dK, dV = (wide[:, o:o + D].unflatten(1, (1, D)) for o in (0, 64, 128, 192))
    tall = torch.empty((m - 1) * (1 << 30) + 1024, dtype=BF16, device=DEV)
    Q, dO, O, dQ = (tall.as_strided((m, 2, D), (1 << 30, D, 1), o) for o in (0, 128, 256, 384))
    guard = [wide[:, o:o + 16] for o in (32, 96, 160, 224)] + [tall.as_strided((m, 32), (1 << 30, 1), o) for o in (64, 192, 320, 448)]
    for t in guard:
        t.fill_(7)
    for t, x in ((K, p.K), (V, p.V), (Q, p.Q), (dO, p.dO)):
        t.copy_(x.to(DEV))
    o = p.options(DEV)
    _, lse = sp.sp_attention(S, Q, K, V, O=O, **o)
    _, _, _, dT = sp.sp_attention_grad(S, Q, K, V, O, lse, dO, dQ=dQ, dK=dK, dV=dV, **o)
    ref = reference(p)
    check({"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV, **({"dT": dT} if buckets else {})}, ref)
    assert all(bool((t == 7).all()) for t in guard)
