"""sp_attention and sp_attention_grad against the definition in 64 bits (tests/attention_util.py, which also derives the bounds), through the
C ABI: types, head layouts, lengths, odd sizes, strides, rows that attend to nothing, the position bias, the inspector's choices."""
import pytest
import torch

import paper_2202_04305_amd as sp
from attention_util import Problem, reference
from gpu_util import say, DEV

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def pack(at, lt=(0, 1), pw=32, cw=32):
    rows, cols = at.nonzero(as_tuple=True)
    enc = sp.sp_encode(lt, (0, 1), pw, cw)
    vals = torch.zeros(rows.numel(), dtype=torch.float32, device=DEV)          # the values play no part
    return sp.sp_pack(enc, tuple(at.shape), [rows.to(DEV).contiguous(), cols.to(DEV).contiguous()], vals)


def problem(at, H, Hk, D, dt, seed=0, buckets=0, positions=None, train=True, **more):
    g = torch.Generator().manual_seed(1000 + seed)
    m, n = at.shape

    def draw(rows, heads):
        return torch.randn(rows, heads, D, generator=g).to(dt)
    p = Problem(at, draw(m, H), draw(n, Hk), draw(n, Hk), dO=draw(m, H) if train else None, **more)
    if buckets:
        p.bias = torch.randn(buckets, H, generator=g).to(dt)
    if positions is not None:
        p.qpos, p.kpos = (t.to(torch.int32) for t in positions)
    return p


def run(S, p, grads=True, **outputs):
    o = p.options(DEV)
    Q, K, V = p.Q.to(DEV), p.K.to(DEV), p.V.to(DEV)
    O, lse = sp.sp_attention(S, Q, K, V, **o)
    got = {"O": O, "lse": lse}
    if grads:
        got["dQ"], got["dK"], got["dV"], dT = sp.sp_attention_grad(S, Q, K, V, O, lse, p.dO.to(DEV), **o)
        if dT is not None:
            got["dT"] = dT
    return got


def check(got, ref, what=""):
    torch.cuda.synchronize()
    for k, (want, tol) in ref.items():
        x = got[k].double().cpu()
        assert x.shape == want.shape, (what, k, x.shape, want.shape)
        same = (x == want) | (torch.isnan(x) & torch.isnan(want))
        bad = ~(same | ((x - want).abs() <= tol))
        assert not bad.any(), "%s %s: %d of %d outside, worst %.2f of the bound, first at %s: %s, not %s" % (
            what, k, int(bad.sum()), bad.numel(), float(((x - want).abs() / tol)[bad].max()), bad.nonzero()[0].tolist(),
            float(x[bad][0]), float(want[bad][0]))


def check_all(at, H, Hk, D, dt, grads=True, lt=(0, 1), pw=32, cw=32, **more):
    p = problem(at, H, Hk, D, dt, **more)
    S = sp.sp_prepare_attention(pack(at, lt, pw, cw), grad=grads)
    check(run(S, p, grads), reference(p, grads), "%s H %d/%d D %d %s" % (tuple(at.shape), H, Hk, D, dt))
    return S


def ragged(lq, lk):
    """A batch: a rectangle of queries times keys for each sequence."""
    at = torch.zeros(sum(lq), sum(lk), dtype=torch.bool)
    i = j = 0
    for a, b in zip(lq, lk):
        at[i:i + a, j:j + b] = True
        i, j = i + a, j + b
    return at


def band(m, n, width, everyone=0):
    i, j = torch.arange(m)[:, None], torch.arange(n)[None, :]
    return ((i - j).abs() <= width) | (j < everyone)


def random_pattern(m, n, share, seed=0):
    return torch.rand(m, n, generator=torch.Generator().manual_seed(seed)) < share


PATTERNS = {
    "one pair": lambda: torch.ones(1, 1, dtype=torch.bool),
    "one row": lambda: torch.ones(1, 200, dtype=torch.bool),
    "one column": lambda: torch.ones(150, 1, dtype=torch.bool),
    "dense": lambda: torch.ones(130, 193, dtype=torch.bool),
    "ragged batch": lambda: ragged([1, 37, 128, 5, 60], [64, 0, 130, 1, 77]),
    "band": lambda: band(300, 300, 20, 3),
    "sparse": lambda: random_pattern(200, 500, 0.02),
    "half": lambda: random_pattern(140, 150, 0.5),
    "empty rows": lambda: random_pattern(100, 90, 0.3) & (torch.arange(100) % 3 == 1)[:, None],
    "tokens behind a prefix": lambda: torch.cat([torch.ones(40, 150, dtype=torch.bool), ragged([1] * 40, list(range(40)))], 1),
    "nothing stored": lambda: torch.zeros(20, 30, dtype=torch.bool),
}


@pytest.mark.parametrize("name", PATTERNS)
@pytest.mark.parametrize("dt", [BF16, F32])
def test_patterns(name, dt):
    say("case", name, dt)
    check_all(PATTERNS[name](), 4, 2, 64, dt)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("D", [1, 7, 8, 31, 32, 40, 64, 80, 100, 128, 136, 192, 256])
def test_head_sizes(D, dt):
    say("case head size", D, dt)
    if dt == F32 and D > 128:                            # does not fit a lane's registers: refused
        with pytest.raises(sp.SpError):
            check_all(ragged([70, 33], [65, 100]), 2, 1, D, dt)
        return
    check_all(ragged([70, 33], [65, 100]), 2, 1, D, dt)
    check_all(ragged([1, 1, 1], [300, 17, 64]), 2, 2, D, dt)
    # with a bias: rows of blocks, single rows, few rows of many heads
    where = dict(positions=(torch.arange(103) + 20, torch.arange(165)), buckets=32, causal=True, bidirectional=False)
    check_all(ragged([70, 33], [65, 100]), 2, 1, D, dt, **where)
    check_all(ragged([70, 33], [65, 100]), 8, 1, D, dt, **where)
    check_all(ragged([1, 1, 1], [300, 17, 64]), 2, 2, D, dt, positions=(torch.tensor([200, 10, 60]), torch.arange(381)), buckets=64, max_distance=200)
    check_all(torch.ones(9, 400, dtype=torch.bool), 6, 1, D, dt, positions=(torch.arange(9) * 40, torch.arange(400)), buckets=64, max_distance=200)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("D", [24, 64, 72, 128, 200, 256])
@pytest.mark.parametrize("heads", [(2, 2), (2, 1), (6, 1)])
def test_few_rows_and_few_keys(heads, D, dt):
    """Blocks of 32 rows, and of 32 keys, over long stretches of the other side that are cut into several items."""
    if dt == F32 and D > 128:
        pytest.skip("refused: does not fit a lane's registers")
    say("case few", heads, D, dt)
    g = torch.Generator().manual_seed(D)
    for m, n in ((20, 700), (700, 20)):
        at = torch.rand(m, n, generator=g) < 0.8
        check_all(at, heads[0], heads[1], D, dt)
        check_all(at, heads[0], heads[1], D, dt, buckets=32, positions=(torch.arange(m) * 3, torch.arange(n) * 2 - 40), causal=D % 16 == 0, bidirectional=D != 64)


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (3, 1), (6, 2), (8, 8), (8, 1), (40, 1), (70, 2)])
@pytest.mark.parametrize("name", ["one row", "ragged batch", "band", "sparse", "tokens behind a prefix"])
def test_head_layouts(name, heads):
    say("case heads", name, heads)
    check_all(PATTERNS[name](), heads[0], heads[1], 32, BF16)


@pytest.mark.parametrize("lt,pw,cw", [((1, 1), 32, 32), ((0, 1), 64, 64), ((1, 1), 64, 64), ((0, 1), 32, 64), ((0, 1), 64, 32), ((0, 1), 16, 8), ((1, 1), 16, 16)])
def test_encodings_and_widths(lt, pw, cw):
    """Rows that DCSR does not store get zeros; narrow widths have 32-bit working copies, wide ones are narrowed by the inspector."""
    say("case encoding", lt, pw, cw)
    check_all(random_pattern(90, 100, 0.2) & (torch.arange(90) % 4 == 2)[:, None], 2, 1, 64, BF16, lt=lt, pw=pw, cw=cw)
    check_all(random_pattern(90, 100, 0.01), 2, 1, 64, F32, lt=lt, pw=pw, cw=cw)


def test_many_columns_and_windows():
    """More columns than a window of the inspector, far apart, with rows that meet in some of them."""
    m, n = 70, 60000
    at = torch.zeros(m, n, dtype=torch.bool)
    g = torch.Generator().manual_seed(5)
    at[:, [0, 31, 32, 8191, 8192, 16383, 16384, 59999]] = True
    at[torch.randint(m, (500,), generator=g), torch.randint(n, (500,), generator=g)] = True
    at[3] = False
    check_all(at, 2, 2, 32, BF16)


@pytest.mark.parametrize("m,n", [(0, 5), (5, 0), (0, 0)])
def test_empty_shapes(m, n):
    p = problem(torch.zeros(m, n, dtype=torch.bool), 2, 1, 16, BF16)
    enc = sp.sp_encode((0, 1), (0, 1), 32, 32)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    S = sp.sp_prepare_attention(sp.sp_pack(enc, (m, n), [none, none], torch.zeros(0, device=DEV)), grad=True)
    got = run(S, p)
    torch.cuda.synchronize()
    assert got["O"].shape == (m, 2, 16) and not got["O"].any() and bool((got["lse"] == float("-inf")).all())
    assert not got["dQ"].any() and not got["dK"].any() and not got["dV"].any()


POSITIONS = {
    "both directions": dict(bidirectional=True, causal=False),
    "backwards only": dict(bidirectional=False, causal=False),
    "backwards, causal": dict(bidirectional=False, causal=True),
    "both directions, causal": dict(bidirectional=True, causal=True),
}


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("kind", POSITIONS)
@pytest.mark.parametrize("buckets,far", [(32, 128), (4, 2), (64, 300), (8, 4096), (22, 50)])
def test_position_bias(kind, buckets, far, dt):
    o = dict(POSITIONS[kind])
    say("case bias", kind, buckets, far, dt)
    if far <= (buckets // 4 if o["bidirectional"] else buckets // 2):
        far = buckets
    at = ragged([70, 40], [90, 45])
    pos = (torch.cat([torch.arange(70) * 3, torch.arange(40) + 500]), torch.cat([torch.arange(90) * 2, torch.arange(45) + 480]))
    check_all(at, 4, 2, 32, dt, buckets=buckets, positions=pos, max_distance=far, **o)


def test_position_bias_with_rows_that_attend_to_everything():
    """A band whose first rows store every column as well: they are cut, their gradients joined."""
    m = 6000
    at = band(m, m, 12)
    at[:3] = True
    at[:, :2] = True
    for dt in (BF16, F32):
        check_all(at, 1, 1, 32, dt, buckets=16, positions=(torch.arange(m), torch.arange(m)), max_distance=40)


@pytest.mark.parametrize("name", ["one row", "band", "sparse", "tokens behind a prefix"])
def test_position_bias_by_pattern(name):
    at = PATTERNS[name]()
    say("case bias", name)
    for heads in ((2, 2), (6, 1), (40, 1)):
        check_all(at, heads[0], heads[1], 64, BF16, buckets=32, positions=(torch.arange(at.shape[0]) + 100, torch.arange(at.shape[1])))


def test_positions_at_the_ends_of_their_type():
    at = torch.ones(3, 4, dtype=torch.bool)
    lo, hi = -2 ** 31, 2 ** 31 - 1
    pos = (torch.tensor([lo, 0, hi]), torch.tensor([lo, hi, 0, 5]))
    for causal in (False, True):
        check_all(at, 2, 2, 16, F32, buckets=8, positions=pos, max_distance=64, causal=causal)


def test_causal_without_bias_and_rows_that_it_empties():
    at = torch.ones(100, 130, dtype=torch.bool)
    pos = (torch.arange(100) - 20, torch.arange(130))
    for dt in (BF16, F32):
        check_all(at, 2, 1, 64, dt, positions=pos, causal=True)


def test_lowest_and_infinite_biases():
    """A bucket of the type's lowest value or minus infinity leaves its pairs without weight; a row of nothing else gives zero."""
    for dt in (BF16, F16, F32):
        for low in (float(torch.finfo(dt).min), float("-inf")):
            at = torch.ones(40, 50, dtype=torch.bool)
            at[7, 3:] = False
            p = problem(at, 2, 1, 32, dt, buckets=4, positions=(torch.arange(40), torch.arange(50)), max_distance=8, bidirectional=False)
            p.bias[0] = low                              # keys at or behind the query
            at[9] = torch.arange(50) >= 9                # the whole row in that bucket
            if low == float("-inf"):
                ref = reference(p)
            else:                                        # the lowest value is a number: a row of nothing else is a row like any other
                p.at[9] = False
                ref = reference(p)
            S = sp.sp_prepare_attention(pack(p.at), grad=True)
            check(run(S, p), ref, "%s %s" % (dt, low))


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", ["band", "sparse", "ragged batch", "tokens behind a prefix"])
def test_what_a_row_does_not_attend_to_has_no_influence(name, bad, dt):
    """A key and value of NaN / infinity reach the rows that store them and no others, whichever rows they share a block with."""
    at = PATTERNS[name]()
    p = problem(at, 2, 1, 32, dt, train=False)
    col = int(at.sum(0).argmin()) if name != "tokens behind a prefix" else at.shape[1] - 1
    p.K[col], p.V[col] = bad, bad
    say("case", name, bad, dt, "rows", int(at[:, col].sum()))
    S = sp.sp_prepare_attention(pack(at))
    got = run(S, p, False)
    clean = ~at[:, col]
    p.K[col], p.V[col] = 0, 0
    ref = reference(p, False)
    check({"O": got["O"][clean.to(DEV)], "lse": got["lse"][:, clean.to(DEV)]},
          {"O": tuple(t[clean] for t in ref["O"]), "lse": tuple(t[:, clean] for t in ref["lse"])}, name)
    assert bool(torch.isnan(got["O"][(~clean).to(DEV)]).all())


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("name", ["band", "ragged batch"])
def test_gradients_of_rows_beside_one_that_is_not_a_number(name, dt):
    """A query (and its dO) of NaN spoils its own gradient and those of the keys that it attends to; all other gradients stay right."""
    at = PATTERNS[name]()
    p = problem(at, 2, 1, 32, dt)
    row = 30
    S = sp.sp_prepare_attention(pack(at), grad=True)
    p.Q[row], p.dO[row] = float("nan"), float("nan")
    got = run(S, p)
    p.Q[row], p.dO[row] = 0, 0
    at2 = p.at.clone()
    p.at = at2
    at2[row] = False
    ref = reference(p)
    rows, cols = torch.arange(at.shape[0]) != row, ~at[row]
    check({"dQ": got["dQ"][rows.to(DEV)], "dK": got["dK"][cols.to(DEV)], "dV": got["dV"][cols.to(DEV)]},
          {"dQ": tuple(t[rows] for t in ref["dQ"]), "dK": tuple(t[cols] for t in ref["dK"]), "dV": tuple(t[cols] for t in ref["dV"])}, name)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_strides(dt):
    """Heads before tokens, a slice of a wider row, a start that is not 16-byte aligned, one K and V for all heads by a stride of zero."""
    at = ragged([50, 20], [60, 70])
    p = problem(at, 4, 2, 40, dt)
    ref = reference(p)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    o = p.options(DEV)

    def heads_first(t):
        return t.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)

    def in_wider(t, shift):
        w = torch.full((t.shape[0], t.shape[1], t.shape[2] + 9), float("nan"), dtype=dt, device=DEV)
        v = w[:, :, shift:shift + t.shape[2]]
        v.copy_(t)
        return v
    for name, lay in (("heads first", heads_first), ("shifted by 8", lambda t: in_wider(t, 8)), ("shifted by 1", lambda t: in_wider(t, 1))):
        Q, K, V, dO = (lay(t) for t in (p.Q, p.K, p.V, p.dO))
        outs = {k: lay(torch.zeros_like(t)) for k, t in (("O", p.Q), ("dQ", p.Q), ("dK", p.K), ("dV", p.V))}
        O, lse = sp.sp_attention(S, Q, K, V, O=outs["O"], **o)
        sp.sp_attention_grad(S, Q, K, V, O, lse, dO, dQ=outs["dQ"], dK=outs["dK"], dV=outs["dV"], **o)
        check({**outs, "lse": lse}, ref, name)
        if name.startswith("shifted"):                   # nothing beside the rows was written
            for t in outs.values():
                whole = t._base
                assert int(torch.isnan(whole).sum()) == whole.shape[0] * whole.shape[1] * 9, name
    p.K, p.V = p.K[:, :1].expand(-1, 4, -1), p.V[:, :1].expand(-1, 4, -1)
    got, _ = sp.sp_attention(S, p.Q.to(DEV), p.K[:, :1].contiguous().to(DEV).expand(-1, 4, -1), p.V[:, :1].contiguous().to(DEV).expand(-1, 4, -1), **o)
    check({"O": got}, {"O": reference(p, False)["O"]}, "expanded")


def test_decoding_steps_over_caches_from_one_recorded_graph():
    """Serving: a pattern with room for 40 tokens of each sequence is packed once; a recorded step appends a key and value where its positions
    say and attends with bias and causal.  The caches' free places hold NaN.  Then cross attention to states of another length."""
    B, room, H, Hk, D = 3, 40, 4, 2, 32
    g = torch.Generator().manual_seed(4)
    lens = torch.tensor([5, 0, 30])
    own, cross = ragged([1] * B, [room] * B), ragged([1] * B, [17, 60, 9])
    S, X = (sp.sp_prepare_attention(pack(a)) for a in (own, cross))
    bias = torch.randn(16, H, generator=g).to(BF16)
    K, V = (torch.full((B * room, Hk, D), float("nan"), dtype=BF16) for _ in range(2))
    for b in range(B):
        for t in (K, V):
            t[b * room:b * room + int(lens[b])] = torch.randn(int(lens[b]), Hk, D, generator=g).to(BF16)
    states = [torch.randn(86, Hk, D, generator=g).to(BF16) for _ in range(2)]
    kpos = torch.arange(room, dtype=torch.int32).repeat(B)
    dev = dict(K=K.to(DEV), V=V.to(DEV), q=torch.zeros(B, H, D, dtype=BF16, device=DEV), k=torch.zeros(B, Hk, D, dtype=BF16, device=DEV),
               v=torch.zeros(B, Hk, D, dtype=BF16, device=DEV), pos=lens.int().to(DEV), kpos=kpos.to(DEV), bias=bias.to(DEV))
    base = torch.arange(B, device=DEV) * room
    SK, SV = (t.to(DEV) for t in states)

    def step():
        at = base + dev["pos"]
        dev["K"].index_copy_(0, at, dev["k"])
        dev["V"].index_copy_(0, at, dev["v"])
        O, _ = sp.sp_attention(S, dev["q"], dev["K"], dev["V"], causal=True, qpos=dev["pos"], kpos=dev["kpos"], bias=dev["bias"], max_distance=20, bidirectional=False)
        return O, sp.sp_attention(X, O, SK, SV)[0]
    saved = dev["K"].clone(), dev["V"].clone()
    step()                                               # warm, then as it was
    dev["K"].copy_(saved[0]); dev["V"].copy_(saved[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, Y = step()
    dev["K"].copy_(saved[0]); dev["V"].copy_(saved[1])
    for n in range(6):
        q, k, v = torch.randn(B, H, D, generator=g).to(BF16), torch.randn(B, Hk, D, generator=g).to(BF16), torch.randn(B, Hk, D, generator=g).to(BF16)
        for name, t in (("q", q), ("k", k), ("v", v)):
            dev[name].copy_(t)
        dev["pos"].copy_(lens.int() + n)
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            K[b * room + int(lens[b]) + n], V[b * room + int(lens[b]) + n] = k[b], v[b]
        p = Problem(own, q, torch.nan_to_num(K), torch.nan_to_num(V), causal=True, qpos=lens.int() + n, kpos=kpos, bias=bias, max_distance=20, bidirectional=False)
        check({"O": O}, {"O": reference(p, False)["O"]}, "step %d" % n)
        check({"O": Y}, {"O": reference(Problem(cross, O.cpu(), *states), False)["O"]}, "step %d, cross" % n)


def test_offsets_beyond_32_bits():
    """Rows of K and V so far apart that the last ones lie more than 2^32 bytes, and 2^31 numbers, behind the first."""
    n, ld, D = 150_000, 16_384, 32
    at = torch.zeros(5, n, dtype=torch.bool)
    g = torch.Generator().manual_seed(8)
    at[:, torch.randint(n, (60,), generator=g)] = True
    at[:3, n - 40:] = True
    at[3, :] = False
    p = problem(at, 2, 1, D, BF16, train=False)
    S = sp.sp_prepare_attention(pack(at))
    far = torch.empty(n * ld, dtype=BF16, device=DEV)
    K, V = (far.view(n, ld)[:, o:o + D].unflatten(1, (1, D)) for o in (0, 64))
    K.copy_(p.K.to(DEV))
    V.copy_(p.V.to(DEV))
    assert (n - 1) * K.stride(0) > 2 ** 31
    O, lse = sp.sp_attention(S, p.Q.to(DEV), K, V)
    check({"O": O, "lse": lse}, reference(p, False))


def test_gradients_against_differences():
    """(L(x + h) - L(x - h)) / 2h of L = sum(O * dO), both sides on the GPU in f32 with the sum in f64.  h = 2^-7: the cubic term is of the order
    h^2 = 6e-5 of the gradient's scale, the rounding of O (2^-24 of it, 70 * 6 * 32 numbers) over 2h of the order 1e-4."""
    at = ragged([40, 30], [50, 25])
    p = problem(at, 6, 2, 32, F32, buckets=8, positions=(torch.arange(70), torch.arange(75)), max_distance=40)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got = run(S, p)
    h = 2.0 ** -7
    g = torch.Generator().manual_seed(3)
    for name, grad in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("bias", "dT")):
        x = getattr(p, name)
        along = torch.randn(x.shape, generator=g)
        along /= along.norm()
        ends = []
        for sign in (1, -1):
            setattr(p, name, x + sign * h * along)
            ends.append(float((run(S, p, False)["O"].double().cpu() * p.dO.double()).sum()))
        setattr(p, name, x)
        slope, want = (ends[0] - ends[1]) / (2 * h), float((got[grad].double().cpu() * along.double()).sum())
        assert abs(slope - want) <= 1e-2 * float(got[grad].double().norm()) + 1e-3, (name, slope, want)


def test_same_bits_on_every_call_and_from_a_graph():
    """Long rows that are cut and joined, the bias's gradient, everything recorded: replays give the eager call's bits."""
    cases = [(torch.cat([torch.ones(24, 5000, dtype=torch.bool), ragged([1] * 24, [40] * 24)], 1), 8, 2, 64, BF16, 0),
             (band(700, 700, 64, 5), 4, 4, 64, BF16, 16), (ragged([1] * 5, [3000, 10, 700, 0, 1500]), 4, 4, 128, F32, 0)]
    for at, H, Hk, D, dt, buckets in cases:
        pos = (torch.arange(at.shape[0]), torch.arange(at.shape[1])) if buckets else None
        p = problem(at, H, Hk, D, dt, buckets=buckets, positions=pos)
        S = sp.sp_prepare_attention(pack(at), grad=True)
        eager = run(S, p)
        o = p.options(DEV)
        Q, K, V, dO = (t.to(DEV) for t in (p.Q, p.K, p.V, p.dO))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            O, lse = sp.sp_attention(S, Q, K, V, **o)
            grads = sp.sp_attention_grad(S, Q, K, V, O, lse, dO, **o)
        for rep in range(4):
            for t in (O, lse) + grads:
                if t is not None:
                    t.fill_(7)
            again = run(S, p)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k, t in zip(("O", "lse", "dQ", "dK", "dV", "dT"), (O, lse) + grads):
                if t is not None:
                    assert torch.equal(again[k], eager[k]), (k, rep)
                    assert torch.equal(t, eager[k]), (k, rep)


def test_calls_that_overlap_on_two_streams_and_in_two_graphs():
    at = torch.ones(16, 4000, dtype=torch.bool)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    ps = [problem(at, 8, 2, 64, BF16, seed=s) for s in (1, 2)]
    want = [run(S, p) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    ins = [[t.to(DEV) for t in (p.Q, p.K, p.V, p.dO)] for p in ps]
    torch.cuda.synchronize()
    outs = [[], []]
    for rep in range(10):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                Q, K, V, dO = ins[k]
                O, lse = sp.sp_attention(S, Q, K, V)
                outs[k].append((O, lse) + sp.sp_attention_grad(S, Q, K, V, O, lse, dO)[:3])
    torch.cuda.synchronize()
    for k in range(2):
        for got in outs[k]:
            for name, t in zip(("O", "lse", "dQ", "dK", "dV"), got):
                assert torch.equal(t, want[k][name]), (k, name)
    graphs, made = [], []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            Q, K, V, dO = ins[k]
            O, lse = sp.sp_attention(S, Q, K, V)
            made.append((O, lse) + sp.sp_attention_grad(S, Q, K, V, O, lse, dO)[:3])
        graphs.append(g)
    for rep in range(5):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                graphs[k].replay()
        torch.cuda.synchronize()
        for k in range(2):
            for name, t in zip(("O", "lse", "dQ", "dK", "dV"), made[k]):
                assert torch.equal(t, want[k][name]), (k, name, rep)


def test_scores_then_softmax_then_product_by_the_other_calls():
    """The same attention made of sp_sddmm, a softmax over the stored entries and sp_matmul, for one head in f32."""
    at = random_pattern(120, 150, 0.3)
    p = problem(at, 1, 1, 64, F32, train=False)
    S = sp.sp_prepare_attention(pack(at))
    O, _ = sp.sp_attention(S, p.Q.to(DEV), p.K.to(DEV), p.V.to(DEV))
    rows, cols = at.nonzero(as_tuple=True)
    enc = sp.sp_encode((0, 1), (0, 1), 32, 32)
    place = [rows.to(DEV).contiguous(), cols.to(DEV).contiguous()]
    ones = sp.sp_pack(enc, at.shape, place, torch.ones(rows.numel(), device=DEV))
    s = sp.sp_sddmm(ones, p.Q[:, 0].to(DEV).contiguous(), p.K[:, 0].to(DEV).contiguous(), b_is_transposed=True).double() * p.scale
    dense = torch.full(at.shape, float("-inf"), dtype=torch.float64, device=DEV)
    dense[place[0], place[1]] = s
    w = torch.softmax(dense, 1).nan_to_num(0)[place[0], place[1]].float()
    out = sp.sp_matmul(sp.sp_pack(enc, at.shape, place, w), p.V[:, 0].to(DEV).contiguous(), torch.empty(120, 64, device=DEV))
    ref, tol = reference(p, False)["O"]
    assert bool(((out.double().cpu() - ref[:, 0]).abs() <= 2 * tol[:, 0]).all())
    assert bool(((O[:, 0].double() - out.double()).abs().cpu() <= 3 * tol[:, 0]).all())


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-3, 2.5])
def test_scales(scale, dt):
    """Zero (every pair weighs the same), negative, small and large ones."""
    check_all(ragged([50, 3], [70, 40]), 2, 1, 64, dt, scale=scale)
    check_all(ragged([50, 3], [70, 40]), 2, 1, 64, dt, scale=scale, buckets=8, positions=(torch.arange(53), torch.arange(110)), max_distance=20)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("name", ["band", "sparse", "tokens behind a prefix"])
def test_gradients_of_rows_that_do_not_attend_to_one_that_is_not_a_number(name, dt):
    """A key and value of NaN spoil what attends to them; all other rows' and keys' gradients stay right."""
    at = PATTERNS[name]()
    p = problem(at, 2, 1, 32, dt)
    col = int((at.sum(0) + 1000 * (at.sum(0) == 0)).argmin())
    S = sp.sp_prepare_attention(pack(at), grad=True)
    p.K[col], p.V[col] = float("nan"), float("nan")
    rows = ~at[:, col]
    p.dO[~rows] = 0                                      # those rows' own gradients are lost, and the other keys' share of them
    got = run(S, p)
    p.K[col], p.V[col] = 0, 0
    p.at = at & rows[:, None]
    ref = reference(p)
    keys = ~at[~rows].any(0)
    check({"dQ": got["dQ"][rows.to(DEV)], "dK": got["dK"][keys.to(DEV)], "dV": got["dV"][keys.to(DEV)]},
          {"dQ": tuple(t[rows] for t in ref["dQ"]), "dK": tuple(t[keys] for t in ref["dK"]), "dV": tuple(t[keys] for t in ref["dV"])}, name)


def test_f16_gradients_beyond_the_type():
    """dO so large that ds does not fit f16: such rows are made again pair by pair, in f32."""
    at = ragged([40, 20], [50, 30])
    p = problem(at, 2, 1, 32, F16)
    p.dO[7] = p.dO[7] * 8000
    p.K, p.V = p.K * 0.05, p.V
    S = sp.sp_prepare_attention(pack(at), grad=True)
    got, ref = run(S, p), reference(p)
    assert float(ref["dQ"][0].abs().max()) < 65504 and float(ref["dV"][0].abs().max()) < 65504
    rows = torch.arange(60) != 7
    check({k: got[k] for k in ("O", "lse", "dV")}, {k: ref[k] for k in ("O", "lse", "dV")})
    check({"dQ": got["dQ"]}, {"dQ": ref["dQ"]})
    assert bool(torch.isfinite(got["dK"]).all()) or float(ref["dK"][0].abs().max()) > 65504


def test_inspector_is_refused_while_a_graph_is_recorded():
    at = torch.ones(5, 6, dtype=torch.bool)
    S, T = pack(at), sp.sp_prepare_attention(pack(at))
    x = torch.zeros(4, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        assert code(sp.sp_prepare_attention, S) == 10
        sp.sp_prepare_attention(T)                       # there is nothing left to do
    graph.replay()
    torch.cuda.synchronize()
    assert x.tolist() == [1.0] * 4


def code(f, *a, **k):
    with pytest.raises(sp.SpError) as e:
        f(*a, **k)
    return e.value.code


def test_refusals():
    at = torch.ones(6, 8, dtype=torch.bool)
    p = problem(at, 4, 2, 16, BF16, buckets=8, positions=(torch.arange(6), torch.arange(8)), max_distance=16)
    Q, K, V, dO, T = (t.to(DEV) for t in (p.Q, p.K, p.V, p.dO, p.bias))
    pos = dict(qpos=p.qpos.to(DEV), kpos=p.kpos.to(DEV))
    S = pack(at)
    assert code(sp.sp_attention, S, Q, K, V) == 10                                         # not prepared
    sp.sp_prepare_attention(S)
    O, lse = sp.sp_attention(S, Q, K, V)
    assert code(sp.sp_attention_grad, S, Q, K, V, O, lse, dO) == 10                        # not prepared for gradients
    assert code(sp.sp_attention, S, Q.double(), K.double(), V.double()) == 9
    assert code(sp.sp_attention, S, Q[:, :3], K, V) == 8                                   # 3 heads over 2
    assert code(sp.sp_attention, S, Q, K, V, scale=float("nan")) == 8
    for more in (dict(bias=T[:1]), dict(bias=T[:5]), dict(bias=T, max_distance=2), dict(bias=T, max_distance=5000), dict(bias=T[:0])):
        assert code(sp.sp_attention, S, Q, K, V, **pos, **more) == 8, more
    big = torch.zeros(66, 4, dtype=BF16, device=DEV)
    assert code(sp.sp_attention, S, Q, K, V, bias=big, max_distance=200, **pos) == 8
    wide = torch.zeros(6, 1, 300, dtype=BF16, device=DEV), torch.zeros(8, 1, 300, dtype=BF16, device=DEV)
    assert code(sp.sp_attention, S, wide[0], wide[1], wide[1]) == 8
    for bad in (dict(bias=T), dict(bias=T.float(), **pos), dict(causal=True), dict(causal=True, qpos=pos["kpos"], kpos=pos["kpos"])):
        with pytest.raises(ValueError):
            sp.sp_attention(S, Q, K, V, **bad)
    for q, k, v in ((Q[:5], K, V), (Q, K[:7], V), (Q, K, V[:, :1]), (Q, K.half(), V), (Q, K, V.cpu()), (Q.transpose(1, 2), K, V), (Q[:, 0], K, V)):
        with pytest.raises(ValueError):
            sp.sp_attention(S, q, k, v)
    with pytest.raises(ValueError):
        sp.sp_attention(S, Q, K, V, O=torch.empty(6, 4, 8, dtype=BF16, device=DEV))
    with pytest.raises(ValueError):
        sp.sp_attention(S, Q, K, V, lse=torch.empty(6, 4, device=DEV))
    rows, cols = (t.to(DEV).contiguous() for t in at.nonzero(as_tuple=True))
    vals = torch.zeros(rows.numel(), device=DEV)
    for lt, order in (((0, 1), (1, 0)), ((0, 0), (0, 1)), ((1, 0), (0, 1))):
        assert code(sp.sp_prepare_attention, sp.sp_pack(sp.sp_encode(lt, order, 32, 32), (6, 8), [rows, cols], vals)) == 10
    t3 = sp.sp_pack(sp.sp_encode((0, 1, 1), None, 32, 32), (6, 8, 2), [rows, cols, rows % 2], vals)
    assert code(sp.sp_prepare_attention, t3) == 2
    assert code(sp.sp_attention, t3, Q, K, V) == 2


def test_inspector_out_of_memory_leaves_nothing_behind():
    from paper_2202_04305_amd import binding

    class Metered(binding._TorchAllocator):
        budget = 1 << 30

        def _alloc(self, nbytes, ctx):
            self.budget -= 1
            return super()._alloc(nbytes, ctx) if self.budget >= 0 else None
    at = random_pattern(300, 200, 0.1)
    rows, cols = (t.to(DEV).contiguous() for t in at.nonzero(as_tuple=True))
    alloc = Metered(DEV)
    S = sp.sp_pack(sp.sp_encode((0, 1), None, 32, 32), at.shape, [rows, cols], torch.zeros(rows.numel(), device=DEV), allocator=alloc)
    held, before = len(alloc.live), sp.sp_tensor_info(S).derivedBytes
    for budget in range(200):
        alloc.budget = budget
        try:
            sp.sp_prepare_attention(S, grad=True)
            break
        except sp.SpError as e:
            assert e.code == 12, e
            torch.cuda.synchronize()
    alloc.budget = 1 << 30
    assert budget > 10 and sp.sp_tensor_info(S).derivedBytes > before
    p = problem(at, 2, 2, 32, F32)
    check(run(S, p), reference(p))
    S.free()
    assert len(alloc.live) == 0 and held > 0


@pytest.mark.parametrize("scale", [float("inf"), 3e38, -3e38, 1e300])
def test_scales_without_a_32_bit_value_are_refused(scale):
    """The kernels hold the scale, and its product with log2 e, in 32 bits; the largest of either is 3.4e38."""
    at = torch.ones(6, 8, dtype=torch.bool)
    p = problem(at, 2, 2, 16, BF16)
    S = sp.sp_prepare_attention(pack(at), grad=True)
    Q, K, V, dO = (t.to(DEV) for t in (p.Q, p.K, p.V, p.dO))
    O, lse = sp.sp_attention(S, Q, K, V)
    assert code(sp.sp_attention, S, Q, K, V, scale=scale) == 8
    assert code(sp.sp_attention_grad, S, Q, K, V, O, lse, dO, scale=scale) == 8
