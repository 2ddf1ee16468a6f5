"""The cache held in 4 bits: pages and slots, rows into the pages and back, attention over the pages, and a serving loop of all of them, against
the definitions in 64 bits (tests/cache_util.py, which also derives the bounds)."""
import ctypes
import random

import pytest
import torch

import paper_2202_04305_amd as sp
import cache_util as U
from gpu_util import say, DEV
from paper_2202_04305_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def normal(shape, dt, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt)


# ---- pages and slots --------------------------------------------------------------------------------------------------------

def check_map(lengths, added, free, taken, table, P, pages, tokens, what=""):
    want = U.mapped(lengths, added, free, taken, table, P, pages, tokens)
    t = table.to(DEV)
    got = sp.sp_cache_map(ints(lengths).to(DEV), ints(added).to(DEV), ints(free).to(DEV), ints([taken]).to(DEV), t, P, pages, tokens)
    torch.cuda.synchronize()
    for name, x in zip(("lengths", "start", "position", "slot", "taken", "table"), got + (t,)):
        assert torch.equal(x.cpu(), want[name]), (what, name, x.cpu()[:40], want[name][:40])


def requests(R, longest, most, P, seed, spare=2):
    """Requests with pages of their own, and a list of the rest."""
    r = random.Random(seed)
    lengths, added = [r.choice([0, 1, P - 1, P, P + 1, r.randint(0, longest)]) for _ in range(R)], [r.choice([0, 1, r.randint(0, most)]) for _ in range(R)]
    need = [-(-(a + b) // P) for a, b in zip(lengths, added)]
    pages = sum(need) + spare
    order = list(range(pages))
    r.shuffle(order)
    table = torch.full((R, max(need + [1]) + 1), -1, dtype=torch.int32)
    for k, x in enumerate(lengths):
        for j in range(-(-x // P)):
            table[k, j] = order.pop()
    return lengths, added, order, table, pages


@pytest.mark.parametrize("R,longest,most", [(1, 5, 1), (3, 100, 40), (64, 200, 3), (65, 300, 200), (200, 50, 1), (1000, 400, 30), (5, 20, 20000)])
@pytest.mark.parametrize("P", [16, 64, 48])
def test_map(R, longest, most, P):
    say("case map", R, longest, most, P)
    for seed in (1, 2):
        lengths, added, free, table, pages = requests(R, longest, most, P, seed)
        for tokens in (sum(added), sum(added) + 77, max(0, sum(added) - 5)):
            check_map(lengths, added, free, 0, table, P, pages, tokens, (seed, tokens))
        check_map(lengths, added, [0, 0, 0] + free, 3, table, P, pages, sum(added))


def test_map_where_something_ends():
    table = ints([[4, -1], [5, 6]])
    check_map([10, 20], [30, 40], [0, 1, 2, 3, 7], 0, table, 16, 8, 70, "the table's rows")
    check_map([10, 20], [30, 40], [0, 1], 0, ints([[4, -1, -1, -1], [5, 6, -1, -1]]), 16, 8, 80, "the list")
    check_map([10, 20], [30, 40], [0, 1], 2, ints([[4, -1, -1, -1], [5, 6, -1, -1]]), 16, 8, 80, "the list, all of it taken")
    check_map([10, 20], [30, 40], [0, 1, 2], -2, ints([[4, -1, -1, -1], [5, 6, -1, -1]]), 16, 8, 80, "before the list")
    check_map([10, 20], [30, 40], [0, 99, -3, 1, 7], 0, ints([[4, -1, -1, -1], [8, 1 << 30, -1, -1]]), 16, 8, 80, "pages that do not exist")
    check_map([-5, 20], [3, -7], [0, 1], 0, ints([[4, -1], [5, 6]]), 16, 8, 9, "negative numbers")
    check_map([0, 0], [0, 0], [], 0, torch.zeros(2, 0, dtype=torch.int32), 16, 8, 4, "nothing")
    check_map([], [], [3], 1, torch.zeros(0, 4, dtype=torch.int32), 16, 8, 3, "no requests")


def test_map_leaves_the_rest_of_the_table():
    whole = torch.full((3, 9), -77, dtype=torch.int32)
    t = whole.to(DEV)
    sp.sp_cache_map(ints([1, 17, 0]).to(DEV), ints([1, 20, 16]).to(DEV), ints([5, 6, 7]).to(DEV), ints([0]).to(DEV), t[:, 2:6], 16, 8, 37)
    whole[1, 4], whole[2, 2] = 5, 6
    assert torch.equal(t.cpu(), whole)


def test_map_in_a_graph_goes_on_from_replay_to_replay():
    R, P, pages = 5, 16, 200
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(0)).tolist()
    lengths, taken, table = ints([0] * R).to(DEV), ints([0]).to(DEV), torch.full((R, 40), -1, dtype=torch.int32, device=DEV)
    added, free = ints([1] * R).to(DEV), ints(order).to(DEV)
    sp.sp_cache_map(lengths, added, free, taken, table.clone(), P, pages, 64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sp.sp_cache_map(lengths, added, free, taken, table, P, pages, 64)
        lengths.copy_(out[0])
        taken.copy_(out[4])
    now, used, host = [0] * R, 0, torch.full((R, 40), -1, dtype=torch.int32)
    for k in range(6):
        more = [k, 1, 0, 7 * k % 9, 20]
        added.copy_(ints(more))
        graph.replay()
        torch.cuda.synchronize()
        want = U.mapped(now, more, order, used, host, P, pages, 64)
        for name, x in zip(("lengths", "start", "position", "slot", "taken"), out):
            assert torch.equal(x.cpu(), want[name]), (k, name)
        assert torch.equal(table.cpu(), want["table"])
        now, used, host = want["lengths"].tolist(), int(want["taken"]), want["table"]


def test_map_refused_arguments():
    a, t = ints([1, 2]).to(DEV), torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    one = a[:1].clone()
    for args in ((a.long(), a, a, one, t), (a, one, a, one, t), (a, a, a.cpu(), one, t), (a, a, a, a, t), (a, a, a, one, t.long()), (a, a, a, one, t[:1]),
                 (a, a, a, one, torch.zeros(4, 2, dtype=torch.int32, device=DEV).t())):
        with pytest.raises(ValueError):
            sp.sp_cache_map(*args, 16, 8, 3)
    for more in ((20, 8, 3), (16, -1, 3), (16, 1 << 27, 3), (0, 8, 3)):
        with pytest.raises(sp.SpError):
            sp.sp_cache_map(a, a, a, one, t, *more)
    with pytest.raises(sp.SpError):                      # rows of the table that would be written over each other
        sp.sp_cache_map(a, a, a, one, t[:1].expand(2, 4), 16, 8, 3)


# ---- rows into the pages and back -------------------------------------------------------------------------------------------

def same(x, want, dt):
    w = want.to(dt)
    return bool(((x.cpu() == w) | (torch.isnan(x.cpu()) & torch.isnan(w))).all())


def rows_of(n, G, d, dt, seed):
    """Rows of every size of number, some blocks of which are zero."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, G, d, generator=g) * torch.exp2(torch.randint(-12, 12, (n, G, 1), generator=g).float())
    return (x * (torch.rand(n, G, d, generator=g) < 0.9)).to(dt)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("d", [1, 16, 31, 32, 33, 40, 64, 80, 96, 100, 128, 160, 192, 250, 256])
def test_store_and_load(d, dt):
    say("case store", d, dt)
    for n, G, P in ((1, 1, 16), (37, 3, 16), (100, 2, 64), (70, 2, 48)):
        pages = 2 * n // P + 3
        c = sp.sp_cache(pages, P, G, d)
        assert (c.pages, c.page_tokens, c.kv_heads, c.head_dim) == (pages, P, G, d)
        K, V = rows_of(n, G, d, dt, 1), rows_of(n, G, d, dt, 2)
        slots = torch.randperm(pages * P, generator=torch.Generator().manual_seed(3))[:n].int()
        if n == 100:                                     # neighbours, from the middle of a page on
            slots = torch.arange(n).int() + 29
        sp.sp_cache_store(c, K.to(DEV), V.to(DEV), slots.to(DEV))
        k, v = sp.sp_cache_load(c, slots.to(DEV), F32)
        assert same(k, U.held(K), F32) and same(v, U.held(V), F32), (n, G, P)
        k, v = sp.sp_cache_load(c, slots.to(DEV), dt)
        assert same(k, U.held(K), dt) and same(v, U.held(V), dt)
        # others hold what they held, and storing what is held changes nothing
        rest = torch.ones(pages * P, dtype=torch.bool)
        rest[slots.long()] = False
        rest = rest.nonzero()[:, 0].int()
        k, v = sp.sp_cache_load(c, rest.to(DEV), BF16)
        assert (k == 0).all() and (v == 0).all()
        before = c.data.clone()
        k, v = sp.sp_cache_load(c, slots.to(DEV), F32)
        sp.sp_cache_store(c, k, v, slots.to(DEV))
        k2, v2 = sp.sp_cache_load(c, slots.to(DEV), F32)
        assert torch.equal(k, k2) and torch.equal(v, v2) and c.data.numel() == before.numel()


def test_every_border_between_numbers():
    """Ties and their neighbours, at every power of two that a type has."""
    y = torch.tensor([b + e for b in (0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.99) for e in (-2.0 ** -9, 0.0, 2.0 ** -9)])
    for dt, powers in ((F32, range(-126, 126)), (BF16, range(-126, 126)), (F16, range(-14, 13))):
        x = torch.stack([torch.cat([y, torch.tensor([top, -top])]) * 2.0 ** e for e in powers for top in (7.0, 6.5, 3.6)]).to(dt)[:, None]
        x = torch.cat([x, -x], 1)
        c, at = sp.sp_cache(-(-len(x) // 16), 16, 2, 32), torch.arange(len(x), dtype=torch.int32, device=DEV)
        sp.sp_cache_store(c, x.to(DEV), x.flip(-1).to(DEV), at)
        k, v = sp.sp_cache_load(c, at, F32)
        assert same(k, U.held(x), F32) and same(v, U.held(x).flip(-1), F32), dt


def test_numbers_that_are_not_finite_and_the_largest():
    for dt in (F32, F16, BF16):
        K, V = rows_of(20, 2, 70, dt, 1), rows_of(20, 2, 70, dt, 2)
        K[3, 1, 40], K[4, 0, 69], V[5, 0, 0], V[6, 1, 33] = float("nan"), float("inf"), -float("inf"), float("nan")
        K[7], V[8], K[9, 0, :] = torch.finfo(dt).max, -torch.finfo(dt).max, torch.finfo(dt).tiny
        V[9] = torch.finfo(dt).tiny * torch.finfo(dt).eps        # the least there is
        c, at = sp.sp_cache(2, 16, 2, 70), torch.arange(20, dtype=torch.int32, device=DEV)
        sp.sp_cache_store(c, K.to(DEV), V.to(DEV), at)
        k, v = sp.sp_cache_load(c, at, F32)
        assert same(k, U.held(K), F32) and same(v, U.held(V), F32)
        assert int(torch.isnan(k).sum()) == 32 + 6 and int(torch.isnan(v).sum()) == 64


def test_slots_that_do_not_exist_and_layouts():
    n, G, d, P, pages = 50, 2, 64, 16, 4
    for dt in (BF16, F32):
        K, V = rows_of(n, G, d, dt, 1), rows_of(n, G, d, dt, 2)
        slots = torch.randperm(pages * P, generator=torch.Generator().manual_seed(1))[:n].int()
        slots[[3, 10, 20, 30]] = ints([-1, pages * P, -2 ** 31, 2 ** 31 - 1])
        guard = torch.full((1 << 16,), 0xAB, dtype=torch.uint8, device=DEV)
        c = sp.sp_cache(pages, P, G, d)
        wide = torch.full((n, G, 100), 7.0, dtype=dt, device=DEV)               # strides, and addresses that are not aligned
        wide[:, :, 3:3 + d] = K.to(DEV)
        turned = V.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)
        sp.sp_cache_store(c, wide[:, :, 3:3 + d], turned, slots.to(DEV))
        there = ((slots >= 0) & (slots < pages * P))[:, None, None]
        out = torch.full((n, G, 100), 9.0, dtype=dt, device=DEV)
        k, v = sp.sp_cache_load(c, slots.to(DEV), dt, K=out[:, :, 5:5 + d])
        assert same(k, torch.where(there, U.held(K), 0.0), dt) and same(v, torch.where(there, U.held(V), 0.0), dt)
        assert (out[:, :, :5] == 9).all() and (out[:, :, 5 + d:] == 9).all() and (guard == 0xAB).all()
        one = K[:1].to(DEV).expand(n, G, d)              # the same row for every token
        sp.sp_cache_store(c, one, one, slots.to(DEV))
        assert same(sp.sp_cache_load(c, slots.to(DEV), dt)[0], torch.where(there, U.held(K[:1]).expand(n, G, d), 0.0), dt)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("d", [40, 96, 128])
def test_stored_again_the_bytes_stay(d, dt):
    """What is held is stored as it is held, bit for bit: a block's largest number is 4 or 6 times its power of two (or the block is at the least one)."""
    say("case stored again", d, dt)
    n, G, P, pages = 100, 2, 64, 5
    c, slots = sp.sp_cache(pages, P, G, d), torch.randperm(pages * P, generator=torch.Generator().manual_seed(3))[:n].int().to(DEV)
    sp.sp_cache_store(c, rows_of(n, G, d, dt, 1).to(DEV), rows_of(n, G, d, dt, 2).to(DEV), slots)
    before = c.data.clone()
    assert before.any()
    k, v = sp.sp_cache_load(c, slots, F32)
    sp.sp_cache_store(c, k, v, slots)
    assert torch.equal(c.data, before)
    sp.sp_cache_store(c, v, k, slots)
    assert not torch.equal(c.data, before)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("d", [33, 64, 128])
def test_what_lies_beside_the_pages(d, dt):
    """A cache in the middle of other memory: rows for slots that do not exist go nowhere, those that do only into their own page."""
    say("case beside the pages", d, dt)
    n, G, P, pages = 64, 2, 16, 4
    page = sp.sp_cache(1, P, G, d).data.numel()
    before, size = 1 << 16, pages * page
    whole = torch.full((before + size + (1 << 16),), 0xAB, dtype=torch.uint8, device=DEV)
    inside = whole[before:before + size]
    assert inside.data_ptr() % 256 == 0
    c = sp.Cache(inside, B.SpCache(inside.data_ptr(), pages, P, G, d))
    K, V = rows_of(n, G, d, dt, 1), rows_of(n, G, d, dt, 2)
    outside = ints([-1, -2, -16, -17, -64, -2 ** 31, 64, 65, 79, 80, 127, 128, 4096, 2 ** 31 - 1] * 5)[:n]
    sp.sp_cache_store(c, K.to(DEV), V.to(DEV), outside.to(DEV))
    assert (whole == 0xAB).all()
    slots = torch.where(torch.arange(n) % 3 == 0, outside, torch.arange(n).int() % 16 + 32)     # page 2 alone
    slots[torch.arange(n) >= 16] = -1
    sp.sp_cache_store(c, K.to(DEV), V.to(DEV), slots.to(DEV))
    assert (whole[:before + 2 * page] == 0xAB).all() and (whole[before + 3 * page:] == 0xAB).all() and not (inside[2 * page:3 * page] == 0xAB).all()
    k, v = sp.sp_cache_load(c, slots.to(DEV), F32)
    there = (slots >= 32)[:, None, None] & (slots < 48)[:, None, None]
    assert same(k, torch.where(there, U.held(K), 0.0), F32) and same(v, torch.where(there, U.held(V), 0.0), F32)


def test_store_refused_arguments():
    c, K, at = sp.sp_cache(4, 16, 2, 64), torch.zeros(3, 2, 64, device=DEV), ints([0, 1, 2]).to(DEV)
    for k, v, s in ((K.half(), K, at), (K, K[:2], at), (K[:, :1], K[:, :1], at), (K[..., :32], K, at), (K, K, at.long()), (K, K, at[:2]), (K, K, at.cpu()),
                    (K.cpu(), K, at), (torch.zeros(3, 2, 128, device=DEV)[..., ::2], K, at)):
        with pytest.raises(ValueError):
            sp.sp_cache_store(c, k, v, s)
    with pytest.raises(sp.SpError):
        sp.sp_cache_store(c, K.double(), K.double(), at)
    with pytest.raises(sp.SpError):
        sp.sp_cache_load(c, at, torch.float64)
    with pytest.raises(sp.SpError):
        sp.sp_cache_load(c, at, F32, K=torch.zeros(1, 2, 64, device=DEV).expand(3, 2, 64))
    for args in ((4, 20, 2, 64), (4, 16, 0, 64), (4, 16, 2, 257), (-1, 16, 2, 64), (1 << 27, 16, 2, 64)):
        with pytest.raises(sp.SpError):
            sp.sp_cache(*args)
    empty = sp.sp_cache(0, 16, 2, 64)
    sp.sp_cache_store(empty, K, K, at)
    assert (sp.sp_cache_load(empty, at, F32, K=torch.ones_like(K))[0] == 0).all()
    sp.sp_cache_store(c, K[:0], K[:0], at[:0])
    assert sp.sp_cache_load(c, at[:0])[0].shape == (0, 2, 64)


# ---- attention --------------------------------------------------------------------------------------------------------------

class Pages:
    """A cache whose every slot is filled, what it holds in 64 bits, and requests with pages in any order."""

    def __init__(self, lengths, G, d, P, seed=0, spare=2, width=0, K=None, V=None):
        need = [-(-x // P) for x in lengths]
        self.P, self.pages, self.lengths = P, sum(need) + spare, lengths
        n = self.pages * P
        self.K = normal((n, G, d), BF16, seed + 1) if K is None else K(n)
        self.V = normal((n, G, d), BF16, seed + 2) if V is None else V(n)
        self.cache = sp.sp_cache(self.pages, P, G, d)
        self.order = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed + 3)).int()
        self.table = torch.full((len(lengths), max(need + [1, width])), -1, dtype=torch.int32)
        k = 0
        for r, x in enumerate(need):
            self.table[r, :x] = self.order[k:k + x]
            k += x
        self.fill()

    def fill(self):
        sp.sp_cache_store(self.cache, self.K.to(DEV), self.V.to(DEV), torch.arange(len(self.K), dtype=torch.int32, device=DEV))

    def wanted(self, Q, start, **more):
        return U.attended(U.held(self.K), U.held(self.V), Q, self.table, self.lengths, start, self.P, self.pages, **more)

    def run(self, Q, start, **more):
        return dict(zip(("O", "lse"), sp.sp_cache_attention(self.cache, Q.to(DEV), self.table.to(DEV), ints(self.lengths).to(DEV), ints(start).to(DEV), **more)))


def check(got, want, what=""):
    torch.cuda.synchronize()
    for k, (w, tol) in want.items():
        x = got[k].double().cpu()
        assert x.shape == w.shape, (what, k, x.shape, w.shape)
        bad = ~((x == w) | (torch.isnan(x) & torch.isnan(w)) | ((x - w).abs() <= tol))
        assert not bad.any(), "%s %s: %d of %d outside, worst %.2f of the bound, first at %s: %s, not %s" % (
            what, k, int(bad.sum()), bad.numel(), float(((x - w).abs() / tol)[bad].max()), bad.nonzero()[0].tolist(), float(x[bad][0]), float(w[bad][0]))


def starts(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def check_all(lengths, n, H, G, d, dt, P=16, seed=0, scale=None, causal=True, **more):
    p, start = Pages(lengths, G, d, P, seed, **more), starts(n)
    Q = normal((start[-1], H, d), dt, seed + 9)
    check(p.run(Q, start, scale=scale, causal=causal), p.wanted(Q, start, scale=scale, causal=causal), (lengths, n, H, G, d, dt, P))
    return p


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("d", [1, 7, 16, 32, 33, 40, 64, 80, 96, 128, 160, 192, 224, 250, 256])
def test_head_sizes(d, dt):
    say("case head size", d, dt)
    check_all([70, 1, 33, 0, 200], [1] * 5, 4, 2, d, dt)
    check_all([70, 1, 33, 300], [20, 1, 33, 5], 6, 2, d, dt, P=32)
    check_all([150], [150], 2, 1, d, dt, P=64)


@pytest.mark.parametrize("H,G", [(1, 1), (8, 8), (2, 1), (3, 1), (16, 1), (17, 1), (40, 2), (64, 1), (70, 1)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_heads(H, G, dt):
    say("case heads", H, G, dt)
    check_all([100, 17], [1, 1], H, G, 64, dt)
    check_all([100, 17, 40], [3, 17, 9], H, G, 64, dt)
    check_all([130], [70], H, G, 32, dt)


LENGTHS = {
    "one token": ([1], [1]),
    "ends of tiles": ([15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129], [1] * 12),
    "nothing in the cache": ([0, 0, 5], [1, 3, 2]),
    "no queries": ([10, 20, 30, 40], [0, 1, 0, 4]),
    "prompts": ([33, 64, 100], [33, 64, 100]),
    "a piece of a prompt behind a cache": ([500, 300], [130, 65]),
    "mixture": ([700, 20, 333, 64, 1, 900, 15], [1, 20, 1, 64, 1, 128, 3]),
    "more queries than tokens": ([3, 5], [7, 5]),
    "many requests": ([(7 * k) % 90 for k in range(300)], [1 + (k % 5 == 0) * 3 for k in range(300)]),
    "one long one": ([6000, 3], [1, 1]),
    "a long one with many queries": ([3000], [40]),
}


@pytest.mark.parametrize("name", LENGTHS)
@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_lengths(name, dt):
    say("case lengths", name, dt)
    lengths, n = LENGTHS[name]
    check_all(lengths, n, 4, 2, 64, dt)
    check_all(lengths, n, 4, 1, 128, dt, P=64, causal=False, scale=0.2)


@pytest.mark.parametrize("P", [16, 32, 48, 64, 112, 128, 256, 1024])
def test_pages(P):
    say("case pages", P)
    check_all([5, 1000, 257, P, P + 1, P - 1], [1, 1, 4, 1, 17, 2], 8, 2, 96, BF16, P=P)


@pytest.mark.parametrize("length,n,H,G,P", [(40000, 1, 8, 1, 256), (33333, 5, 2, 2, 64), (20001, 600, 1, 1, 128)])
def test_long(length, n, H, G, P):
    say("case long", length, n, H, G, P)
    check_all([length, 50], [n, 1], H, G, 64, BF16, P=P)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_thousands_of_requests(dt):
    """More than 64 times 64 requests, most of one token, with long ones and prompts among them."""
    r = random.Random(5)
    lengths = [r.choice([0, 1, 16, 40]) for _ in range(4500)]
    lengths[7], lengths[2100], lengths[4499] = 3000, 2000, 900
    check_all(lengths, [1] * 4500, 2, 1, 32, dt)
    n = [r.choice([0, 0, 1]) for _ in range(4500)]
    n[100], n[2100], n[4300] = 90, 300, 40
    lengths[100], lengths[4300] = 90, 600
    check_all(lengths, n, 2, 1, 32, dt)
    check_all(lengths, [k and max(k, 30) for k in n[:300]] + [0] * 4200, 2, 2, 32, dt)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_few_tokens_of_each_request(d, dt):
    """Drafted tokens: 17 to 64 columns a request, beside prompts and single tokens, short and over chunks."""
    say("case few tokens", d, dt)
    check_all([300, 33, 8, 1500, 5, 100, 64], [5, 8, 8, 7, 5, 6, 1], 8, 2, d, dt)
    check_all([9000, 30], [6, 200], 4, 1, d, dt, P=64)
    check_all([2000, 700], [33, 16], 2, 2, d, dt, causal=False)


def test_layouts_and_rows_of_no_request():
    """Strides, rows before the first and behind the last request, which stay as they are; lse given and left out."""
    p = Pages([50, 90], 2, 64, 16)
    for dt in (BF16, F32):
        for n in ([4, 30], [1, 1]):
            start = [3, 3 + n[0], 3 + sum(n)]
            m = 40
            Q = normal((m, 4, 64), dt, 5)
            want = p.wanted(Q, start)
            wide = torch.zeros(m, 4, 99, dtype=dt, device=DEV)
            wide[:, :, 1:65] = Q.to(DEV)
            out = torch.full((4, m, 80), 7.0, dtype=dt, device=DEV)
            lse = torch.full((4, m), 7.0, device=DEV)
            got = p.run(wide[:, :, 1:65], start, O=out.transpose(0, 1)[:, :, 8:72], lse=lse)
            rows = slice(start[0], start[2])
            check({"O": got["O"][rows], "lse": got["lse"][:, rows]}, {"O": [t[rows] for t in want["O"]], "lse": [t[:, rows] for t in want["lse"]]})
            keep = torch.ones(m, dtype=torch.bool)
            keep[rows] = False
            assert (out[:, keep] == 7).all() and (lse[:, keep] == 7).all() and (out[..., :8] == 7).all() and (out[..., 72:] == 7).all()
            one = Q[:1].to(DEV).expand(m, 4, 64)         # one row seen as many
            same_rows = p.run(one, start)
            want = p.wanted(Q[:1].expand(m, 4, 64), start)
            check({"O": same_rows["O"][rows]}, {"O": [t[rows] for t in want["O"]]})


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("first", [0, 1, 4, 8])
def test_addresses_moved_by_a_few_numbers(first, dt):
    """Rows of Q, K, V and O at 4, 8, 16 bytes and more from a multiple of 32, heads of 40 next to each other."""
    say("case moved", first, dt)

    def moved(x):
        whole = torch.full((first + x.numel() + 8,), 7.0, dtype=x.dtype, device=DEV)
        view = whole[first:first + x.numel()].view(x.shape)
        view.copy_(x)
        return whole, view
    p, n = Pages([70, 33, 200], 2, 40, 16), [1, 33, 5]
    slots = torch.arange(p.pages * 16, dtype=torch.int32, device=DEV)
    K, V = (moved(x.to(dt))[1] for x in (p.K, p.V))
    sp.sp_cache_store(p.cache, K, V, slots)
    (kw, k), (vw, v) = (moved(torch.zeros(p.K.shape, dtype=dt)) for _ in range(2))
    sp.sp_cache_load(p.cache, slots, dt, K=k, V=v)
    p.K, p.V = p.K.to(dt), p.V.to(dt)
    assert same(k, U.held(p.K), dt) and same(v, U.held(p.V), dt)
    Q = normal((sum(n), 4, 40), dt, 3)
    whole, O = moved(torch.zeros_like(Q))
    check(p.run(moved(Q)[1], starts(n), O=O), p.wanted(Q, starts(n)))
    for w in (kw, vw, whole):
        assert (w[:first] == 7).all() and (w[-8:] == 7).all()


def test_rows_behind_the_last_one():
    """A step that has fewer rows than its requests have queries: those that are there are what they are in the whole step."""
    for n, m in (([20, 30, 5], 33), ([1, 1, 1], 2), ([200, 3, 9], 130)):
        p, start = Pages([300, 200, 50], 2, 64, 16), starts(n)
        Q = normal((start[-1], 4, 64), BF16, 1)
        want = p.wanted(Q, start)
        got = p.run(Q[:m].contiguous(), start)
        check(got, {"O": [t[:m] for t in want["O"]], "lse": [t[:, :m] for t in want["lse"]]}, n)


def test_without_lse_and_refused_workspaces():
    """Through the C ABI: no lse, and a workspace that is missing, too small or not aligned, which leaves O as it was."""
    L = sp.load_library()
    for n in (1, 50):
        p, start = Pages([5000], 2, 64, 64), [0, n]
        Q, table, lengths, begin = normal((n, 8, 64), BF16, 1).to(DEV), p.table.to(DEV), ints([5000]).to(DEV), ints(start).to(DEV)
        O = torch.full_like(Q, 7.0)
        packed = B._PROBLEM.pack(sp.SP_BF16, 8, 1, 0.125, 1, n, Q.data_ptr(), 512, 64, table.data_ptr(), table.shape[1], table.shape[1], lengths.data_ptr(), begin.data_ptr())
        need = ctypes.c_size_t()
        assert L.sp_cache_attention_workspace(p.cache._ref, packed, ctypes.byref(need)) == 0 and need.value > 0
        work = torch.empty(need.value + 256, dtype=torch.uint8, device=DEV)
        stream = torch.cuda.current_stream().cuda_stream

        def call(at, size):
            return L.sp_cache_attention(p.cache._ref, packed, O.data_ptr(), 512, 64, None, at, size, stream)
        assert call(None, need.value) == 1 and call(work.data_ptr(), need.value - 1) == 8 and call(work.data_ptr() + 128, need.value) == 8
        torch.cuda.synchronize()
        assert (O == 7).all()
        assert call(work.data_ptr(), need.value) == 0
        check({"O": O}, {"O": p.wanted(Q.cpu(), start, scale=0.125)["O"]})


def test_pages_that_do_not_exist_are_left_out():
    for n in ([1, 1, 1], [40, 3, 20]):
        p = Pages([200, 100, 60], 2, 64, 16)
        p.table[0, 3], p.table[0, 12], p.table[1, :], p.table[2, 0] = -1, p.pages, -7, 2 ** 31 - 1
        Q = normal((sum(n), 4, 64), BF16, 1)
        check(p.run(Q, starts(n)), p.wanted(Q, starts(n)), n)
        check(p.run(Q, starts(n), causal=False), p.wanted(Q, starts(n), causal=False), n)


def test_lengths_beyond_the_table():
    for n in ([1, 1], [10, 70]):
        p = Pages([40, 100], 1, 32, 16)
        p.lengths = [5000, 2 ** 31 - 1]                  # the table has room for 112
        p.table[p.table < 0] = 1
        Q = normal((sum(n), 2, 32), F32, 1)
        check(p.run(Q, starts(n)), p.wanted(Q, starts(n)), n)
        p.lengths = [-5, 10]
        check(p.run(Q, starts(n)), p.wanted(Q, starts(n)), n)
    p = Pages([40], 1, 32, 16)
    p.table = p.table[:, :0]
    Q = normal((3, 2, 32), F32, 1)
    check(p.run(Q, [0, 3]), p.wanted(Q, [0, 3]))


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("d", [64, 128, 80])
def test_numbers_that_are_not_finite(d, dt):
    """In tokens that rows do not attend to (behind the length, later than the query, other requests) and in tokens that they do."""
    say("case not finite", d, dt)

    def spoilt(tokens):
        def make(n):
            x = normal((n, 2, d), BF16, 17)
            for t, g, k in tokens:
                x[t, g, k] = float("nan") if t % 2 else float("inf")
            return x
        return make
    for lengths, n in (([150, 40, 7], [1, 1, 1]), ([150, 40, 7], [100, 40, 2])):
        plain = Pages(lengths, 2, d, 16)                 # the same pages in the same order, to find the slots

        def slot(r, t):
            return int(plain.table[r, t // 16]) * 16 + t % 16
        behind = [slot(0, 149) // 16 * 16 + 14, slot(1, 39) // 16 * 16 + 8, slot(2, 6) // 16 * 16 + 7, slot(2, 6) // 16 * 16 + 15]
        behind += [s for page in range(plain.pages) if page not in plain.table for s in (page * 16, page * 16 + 5)]
        late = [slot(0, t) for t in (149, 120, 77)] + [slot(1, 20)]
        start = starts(n)
        Q = normal((start[-1], 4, d), dt, 3)
        for name, slots in (("behind", behind), ("attended", late)):
            for where in ("K", "V", "KV"):
                p = Pages(lengths, 2, d, 16, **{w: spoilt([(s, k % 2, (7 * k) % d) for k, s in enumerate(slots)]) for w in where})
                check(p.run(Q, start), p.wanted(Q, start), (name, where, n))
                if name == "behind":
                    assert torch.isfinite(p.run(Q, start)["O"]).all()
    # queries that are not finite, or so large that scores are: their own rows alone
    p = Pages([150, 40], 2, d, 16)
    for n in ([1, 1], [50, 40]):
        start = starts(n)
        Q = normal((start[-1], 4, d), dt, 3)
        Q[0, 1, 3], Q[-1, 2, d - 1] = float("nan"), float("inf")
        got, rest = p.run(Q, start), normal((start[-1], 4, d), dt, 3)
        want = p.wanted(rest, start)
        assert torch.isnan(got["O"][0, 1]).all() and torch.isnan(got["O"][-1, 2]).all() and torch.isnan(got["lse"][1, 0]) and torch.isnan(got["lse"][2, -1])
        for o, w in ((got["O"], want["O"]), (got["lse"].t(), [t.t() for t in want["lse"]])):
            o = o.cpu().clone()
            o[0, 1], o[-1, 2] = w[0][0, 1].to(o.dtype), w[0][-1, 2].to(o.dtype)
            check({"x": o}, {"x": w})


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("d", [16, 33, 64, 80, 128, 250])
def test_requests_cut_into_chunks(d, dt):
    """A table with room for more than 1024 tokens: requests are cut, lengths around the cuts, also where a chunk is left with nothing."""
    say("case chunks", d, dt)
    for n in ([1, 1, 1, 1, 1, 1, 1], [1, 0, 3, 20, 70, 2, 1]):
        start = starts(n)
        p, Q = Pages([255, 256, 257, 300, 1030, 0, 513], 2, d, 16, 5, width=90), normal((start[-1], 6, d), dt, 3)
        check(p.run(Q, start), p.wanted(Q, start), (d, dt, n))


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("d", [64, 128, 80])
def test_numbers_that_are_not_finite_in_chunks(d, dt):
    """In one chunk of several: rows that attend to it lose their result, rows that do not keep theirs; queries that are not finite lose their own rows."""
    say("case chunks, not finite", d, dt)
    lengths = [1500, 300, 700]
    for n in ([1, 1, 1], [100, 40, 2]):
        plain, start = Pages(lengths, 2, d, 16, width=100), starts(n)
        Q = normal((start[-1], 4, d), dt, 3)
        for name, spots in (("late", [(0, 1499), (1, 270)]), ("early", [(0, 3), (2, 600)]), ("a run", [(0, t) for t in range(500, 800)])):
            for where in ("K", "V"):
                def make(tokens):
                    x = normal((tokens, 2, d), BF16, 17)
                    for k, (r, t) in enumerate(spots):
                        x[int(plain.table[r, t // 16]) * 16 + t % 16, k % 2, (7 * k) % d] = float("nan") if k % 3 else float("inf")
                    return x
                p = Pages(lengths, 2, d, 16, width=100, **{where: make})
                check(p.run(Q, start), p.wanted(Q, start), (name, where, n))
        Q[0, 1, 3] = float("nan")
        got, want = plain.run(Q, start), plain.wanted(normal((start[-1], 4, d), dt, 3), start)
        assert torch.isnan(got["O"][0, 1]).all() and torch.isnan(got["lse"][1, 0])
        for o, w in ((got["O"], want["O"]), (got["lse"].t(), [t.t() for t in want["lse"]])):
            o = o.cpu().clone()
            o[0, 1] = w[0][0, 1].to(o.dtype)
            check({"x": o}, {"x": w})


def test_large_and_small_scores():
    """Scores of hundreds to either side, rows whose largest score comes last, a scale of zero, a negative one."""
    for n in ([1, 1], [33, 60]):
        for scale in (0.0, 5.0, -3.0, 40.0):
            for dt in (BF16, F32):
                check_all([300, 60], n, 4, 2, 64, dt, scale=scale, seed=4)

    def rising(count):
        return (torch.arange(count).float()[:, None, None] / 16).expand(count, 1, 32).to(BF16).contiguous()
    for n in (1, 64):
        p = Pages([512], 1, 32, 16, K=rising)
        p.table = torch.arange(32, dtype=torch.int32)[None].contiguous()
        Q = torch.ones(n, 2, 32)
        for scale in (1.0, -1.0):
            check(p.run(Q, [0, n], scale=scale), p.wanted(Q, [0, n], scale=scale))


def test_scores_beyond_f32():
    """Scores of minus infinity weigh nothing; rows of nothing else are rows that attend to nothing; plus infinity is not a number."""
    def huge(count):
        return torch.full((count, 1, 32), 1e38).to(BF16)
    for n in (1, 40):
        p = Pages([64], 1, 32, 16, K=huge)
        Q = torch.full((n, 2, 32), -1e3)
        Q[:, 1] = 1e3
        got = p.run(Q, [0, n], scale=1.0)
        assert (got["O"][:, 0] == 0).all() and (got["lse"][0] == float("-inf")).all()
        assert torch.isnan(got["O"][:, 1]).all() and torch.isnan(got["lse"][1]).all()


def test_chunks_that_weigh_nothing():
    """Scores of minus infinity in whole chunks: what is left decides, and a row of nothing else attends to nothing."""
    def mixed(n):
        x = torch.zeros(n, 1, 32)
        x[:1040] = 1e38
        return x.to(BF16)
    for n in (1, 40):
        for length in (1000, 2000):
            p = Pages([length], 1, 32, 16, K=mixed, spare=128)
            p.table = torch.arange(128, dtype=torch.int32)[None].contiguous()
            got = p.run(torch.full((n, 2, 32), -1e3), [0, n], scale=1.0, causal=False)
            if length < 1040:
                assert (got["O"] == 0).all() and (got["lse"] == float("-inf")).all()
            else:                                        # tokens 1040 to 1999, all of one weight: 960 V of 4 bits, sums of 960 roundings to 32 bits, 3 parts of a weight
                want = U.held(p.V)[1040:length, 0].mean(0)
                assert (got["O"].cpu().double() - want).abs().max() < 2000 * 2.0 ** -24 * U.held(p.V).abs().max()
                assert (got["lse"].cpu() - torch.tensor(960.0).log()).abs().max() < 1e-5          # some 20 roundings of a number below 8


# Requests cut into 5 to 25 chunks, in some of which a column has no weight: lengths, queries, heads, heads of the cache, and pages of the first request's
# table that do not exist.
WEIGHTLESS = {
    "a prompt longer than a chunk": ([2000, 30], [2000, 30], 2, 1, ()),
    "a prompt behind many chunks": ([6000, 50], [300, 50], 2, 1, ()),
    "drafted tokens across a cut": ([1026, 1026, 40], [4, 2, 1], 4, 2, ()),
    "drafted tokens of many heads": ([1026, 1030, 40], [4, 10, 1], 8, 1, ()),
    "drafted tokens behind many chunks": ([6146, 40], [4, 1], 4, 2, ()),
    "missing pages": ([2000, 1300], [1, 1], 4, 2, range(32, 64)),
    "the first pages missing": ([2000, 1300], [1, 1], 4, 2, range(0, 16)),
    "missing pages of many chunks": ([6000, 1300], [1, 1], 4, 2, range(48, 80)),
    "missing pages of a prompt": ([2000, 1300], [40, 70], 4, 1, range(32, 64)),
}


@pytest.mark.parametrize("name", WEIGHTLESS)
@pytest.mark.parametrize("dt", [F32, F16, BF16])
def test_low_scores_beside_chunks_without_weight(name, dt):
    """Scores of -90 to -1000 in the chunks that a row attends to, nothing in the others: those have no say in the row's maximum."""
    say("case low scores", name, dt)
    lengths, n, H, G, gone = WEIGHTLESS[name]

    def positive(count):
        return 1 + normal((count, G, 64), BF16, 31).abs()
    p, start = Pages(lengths, G, 64, 16, 3, width=70, K=positive), starts(n)
    p.table[0, list(gone)] = -1
    Q = -(1 + normal((start[-1], H, 64), F32, 5).abs()) * torch.linspace(1.3, 8, H)[None, :, None]
    Q = Q.to(dt)
    want = p.wanted(Q, start, scale=0.5)
    lse = want["lse"][0]
    assert (lse < -87).all() and (lse > -1000).all()     # the case is what it says
    check(p.run(Q, start, scale=0.5), want, (name, dt))


@pytest.mark.parametrize("lengths,n", [([70, 1500, 300], [1, 1, 1]), ([70, 300], [1, 1]), ([70, 1500], [40, 70]), ([70, 300], [40, 70]), ([6000], [1]), ([700, 30], [300, 6])])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_the_largest_values(lengths, n, dt):
    """Means of values close to the largest that a cache holds are finite, and right, whatever the sums would be."""
    say("case largest values", lengths, n, dt)

    def alike(count):
        return torch.full((count, 2, 64), 2.0 ** 127).to(BF16)

    def mixed(count):
        return (normal((count, 2, 64), F32, 3).clamp(-7, 7) * 2.0 ** 125).to(BF16)

    def sixes(count):
        x = torch.full((count, 2, 64), 6 * 2.0 ** 125)
        x[:, 1, ::2] = -3e-20
        return x.to(BF16)
    start = starts(n)
    Q = normal((start[-1], 4, 64), dt, 9)
    for name, V in (("alike", alike), ("mixed", mixed), ("sixes", sixes)):
        for scale in (0.0, 0.125, 1.0):
            p = Pages(lengths, 2, 64, 16, 1, V=V)
            got, want = p.run(Q, start, scale=scale), p.wanted(Q, start, scale=scale)
            assert torch.isfinite(got["O"]).all(), (name, scale)
            check(got, want, (name, scale))


def test_the_same_bits_every_time_and_other_streams():
    for n in ([1] * 6, [1, 30, 1, 200, 64, 3]):
        p = Pages([3000, 30, 4000, 200, 500, 1000], 2, 128, 64)
        Q, start = normal((sum(n), 8, 128), BF16, 1).to(DEV), starts(n)
        table, lengths, begin = p.table.to(DEV), ints(p.lengths).to(DEV), ints(start).to(DEV)
        first = sp.sp_cache_attention(p.cache, Q, table, lengths, begin)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(3)]
        results = []
        for s in streams:                                # at the same time, each with its own workspace
            with torch.cuda.stream(s):
                results += [sp.sp_cache_attention(p.cache, Q, table, lengths, begin) for _ in range(3)]
        torch.cuda.synchronize()
        for O, lse in results:
            assert torch.equal(O, first[0]) and torch.equal(lse, first[1])


def test_graphs_serve_other_lengths_and_pages():
    P, G, H, d = 16, 2, 8, 64
    for n in ([1, 1, 1], [20, 1, 90]):
        p = Pages([900, 400, 700], G, d, P)
        Q, table, lengths, start = normal((sum(n), H, d), BF16, 1).to(DEV), p.table.to(DEV), ints(p.lengths).to(DEV), ints(starts(n)).to(DEV)
        O, lse = torch.empty_like(Q), torch.empty(H, sum(n), device=DEV)
        graphs = []
        for _ in range(2):                               # two graphs of the same call
            g = torch.cuda.CUDAGraph()
            sp.sp_cache_attention(p.cache, Q, table, lengths, start, O=O, lse=lse)
            torch.cuda.synchronize()
            with torch.cuda.graph(g):
                sp.sp_cache_attention(p.cache, Q, table, lengths, start, O=O, lse=lse)
            graphs.append(g)
        for k, now in enumerate(([900, 400, 700], [100, 333, 20], [899, 0, 1], [500, 401, 699])):
            p.lengths = now
            p.table = p.table.roll(1, 1).clamp(min=0)
            Q.copy_(normal((sum(n), H, d), BF16, 50 + k))
            table.copy_(p.table)
            lengths.copy_(ints(now))
            graphs[k % 2].replay()
            eager = sp.sp_cache_attention(p.cache, Q, table, lengths, start)
            torch.cuda.synchronize()
            assert torch.equal(eager[0], O) and torch.equal(eager[1], lse)
            check({"O": O, "lse": lse}, p.wanted(Q.cpu(), starts(n)), (n, now))


def test_offsets_beyond_32_bits():
    """Pages that lie beyond 2^32 bytes of the cache."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GiB")
    P, G, d = 64, 8, 128
    pages = (5 << 30) // (P * G * 136)
    c = sp.sp_cache(pages, P, G, d)
    assert c.data.numel() > 1 << 32
    for lengths, n in (([150, 70], [1, 1]), ([150, 70], [60, 70])):
        table = ints([[pages - 1, pages - 7, pages - 3], [pages - 2, 0, 5]])
        slots = torch.cat([table[r, :3].long()[:, None] * P + torch.arange(P) for r in range(2)]).reshape(-1)
        K, V = normal((len(slots), G, d), BF16, 1), normal((len(slots), G, d), BF16, 2)
        sp.sp_cache_store(c, K.to(DEV), V.to(DEV), slots.int().to(DEV))
        k, v = sp.sp_cache_load(c, slots.int().to(DEV), F32)
        assert same(k, U.held(K), F32) and same(v, U.held(V), F32)
        Q, start = normal((sum(n), 16, d), BF16, 3), starts(n)
        got = dict(zip(("O", "lse"), sp.sp_cache_attention(c, Q.to(DEV), table.to(DEV), ints(lengths).to(DEV), ints(start).to(DEV))))
        small = ints([[0, 1, 2], [3, 4, 5]])
        check(got, U.attended(U.held(K), U.held(V), Q, small, lengths, start, P, 6))


def test_a_page_beyond_32_bits():
    """Tokens that lie beyond 2^32 bytes of their page: of 16 million zeros before them nothing is left beside scores of 100 and more."""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB")
    P, d = 1 << 24, 256
    c = sp.sp_cache(1, P, 1, d)
    for n in (1, 40):
        length = P - 100 * n
        slots = torch.arange(length - 50, length)
        K, V = 7 + normal((50, 1, d), BF16, 1).abs(), normal((50, 1, d), BF16, n)
        sp.sp_cache_store(c, K.to(DEV), V.to(DEV), slots.int().to(DEV))
        assert same(sp.sp_cache_load(c, slots.int().to(DEV), F32)[1], U.held(V), F32)
        Q = torch.ones(n, 2, d).to(BF16)
        got = sp.sp_cache_attention(c, Q.to(DEV), ints([[0]]).to(DEV), ints([length]).to(DEV), ints([0, n]).to(DEV), causal=False)
        pad = torch.zeros(14, 1, d, dtype=torch.float64)
        want = U.attended(torch.cat([U.held(K), pad]), torch.cat([U.held(V), pad]), Q, torch.tensor([[0, 1, 2, 3]]), [50], [0, n], 16, 4, causal=False)
        assert (want["lse"][0] > 100).all()
        check(dict(zip(("O", "lse"), got)), want)


def test_attention_refused_arguments():
    p = Pages([20, 30], 2, 64, 16)
    Q, table, lengths, start = normal((2, 4, 64), BF16, 1).to(DEV), p.table.to(DEV), ints([20, 30]).to(DEV), ints([0, 1, 2]).to(DEV)
    ok = (p.cache, Q, table, lengths, start)
    for k, bad in ((1, Q[..., :32]), (1, Q.cpu()), (1, Q.transpose(1, 2)), (2, table.long()), (2, table[:1]), (2, table.cpu()), (2, table.t()), (3, lengths.long()),
                   (4, start[:2]), (4, start.long())):
        with pytest.raises(ValueError):
            sp.sp_cache_attention(*ok[:k], bad, *ok[k + 1:])
    for more in (dict(O=Q[:1]), dict(O=Q.float()), dict(lse=torch.zeros(4, 3, device=DEV)), dict(lse=torch.zeros(4, 2, device=DEV).half())):
        with pytest.raises(ValueError):
            sp.sp_cache_attention(*ok, **more)
    for bad in (Q[:, :3], Q.double()):
        with pytest.raises(sp.SpError):
            sp.sp_cache_attention(p.cache, bad, *ok[2:])
    for scale in (float("nan"), 1e300):
        with pytest.raises(sp.SpError):
            sp.sp_cache_attention(*ok, scale=scale)
    with pytest.raises(sp.SpError):
        sp.sp_cache_attention(*ok, O=torch.zeros(1, 4, 64, dtype=BF16, device=DEV).expand(2, 4, 64))
    assert sp.sp_cache_attention(p.cache, Q[:0], table, lengths, ints([0, 0, 0]).to(DEV))[0].shape == (0, 4, 64)
    none = sp.sp_cache_attention(p.cache, Q, table[:0], lengths[:0], start[:1], O=torch.ones_like(Q))
    assert (none[0] == 1).all()


# ---- all of it --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_serving_loop(dt, interleaved):
    """Prompts in pieces and single tokens of requests that come and go: pages and slots from lengths, Q and K turned by their positions, K and V
    into the pages, attention; every step against a plain simulation that keeps every request's rows."""
    R, G, H, d, P, pages = 4, 2, 6, 64, 16, 64
    cache, f = sp.sp_cache(pages, P, G, d), sp.sp_rotary_frequencies(32, factor=4.0, trained=64)
    free = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().to(DEV)
    lengths, taken, table = ints([0] * R).to(DEV), ints([0]).to(DEV), torch.full((R, 12), -1, dtype=torch.int32, device=DEV)
    kept = [[torch.zeros(0, G, d, dtype=torch.float64) for _ in range(2)] for _ in range(R)]
    for step, added in enumerate(([40, 1, 0, 17], [1, 30, 0, 1], [1, 1, 64, 1], [1, 1, 1, 50], [3, 1, 2, 1])):
        n = sum(added)
        rows = n + 3                                     # a padded batch
        Q, K, V = (normal((rows, h, d), dt, 100 * step + k) for k, h in enumerate((H, G, G)))
        lengths, start, position, slot, taken = sp.sp_cache_map(lengths, ints(added).to(DEV), free, taken, table, P, pages, rows)
        q, k = sp.sp_rotary(position, f, Q.to(DEV), K.to(DEV), interleaved=interleaved)
        sp.sp_cache_store(cache, k, V.to(DEV), slot)
        O = torch.full((rows, H, d), 5.0, dtype=dt, device=DEV)
        O, lse = sp.sp_cache_attention(cache, q, table, lengths, start, O=O)
        torch.cuda.synchronize()
        want = [x for r in range(R) for x in range(len(kept[r][0]), len(kept[r][0]) + added[r])]
        assert position.tolist() == want + [-1] * 3 and slot[n:].tolist() == [-1] * 3 and (O[n:] == 5).all()
        at = torch.cat([ints(want), ints([-1] * 3)])
        for x, y in ((Q, q), (K, k)):
            w, tol = U.rotated(x, at, f.cpu(), interleaved)
            assert ((y.double().cpu() - w).abs() <= tol).all()
        begin = starts(added)
        for r in range(R):
            new = slice(begin[r], begin[r + 1])
            kept[r] = [torch.cat([kept[r][0], U.held(k.cpu()[new])]), torch.cat([kept[r][1], U.held(V[new])])]
        # the requests' rows side by side, as if in pages of their own
        width = 12
        side = torch.zeros(R * width * P, G, d, dtype=torch.float64), torch.zeros(R * width * P, G, d, dtype=torch.float64)
        for r in range(R):
            for s, x in zip(side, kept[r]):
                s[r * width * P:r * width * P + len(x)] = x
        want = U.attended(side[0], side[1], q.cpu()[:n], torch.arange(R * width).view(R, width), [len(x[0]) for x in kept], begin, P, R * width)
        check({"O": O[:n], "lse": lse[:, :n]}, want, step)
    assert int(taken) == sum(-(-int(x) // P) for x in lengths)
