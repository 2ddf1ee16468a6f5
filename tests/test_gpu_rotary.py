"""sp_rotary and sp_rotary_grad against the definition in 64 bits (tests/cache_util.py, which also derives the bounds)."""
import pytest
import torch

import paper_2202_04305_amd as sp
from cache_util import rotated
from gpu_util import say, DEV

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def rows(tokens, heads, d, dt, seed=0):
    return torch.randn(tokens, heads, d, generator=torch.Generator().manual_seed(seed)).to(dt)


def close(got, want, tol, what=""):
    torch.cuda.synchronize()
    x = got.double().cpu()
    bad = ~(((x - want).abs() <= tol) | (torch.isnan(x) & torch.isnan(want)) | (x == want))
    assert not bad.any(), "%s: %d of %d outside, first at %s: %s, not %s, bound %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(x[bad][0]), float(want[bad][0]), float(tol[bad][0]))


def places(tokens, most, seed=1):
    return torch.randint(0, most, (tokens,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(1, 0), (2, 2), (64, 64), (64, 32), (128, 128), (80, 20), (80, 80), (96, 40), (128, 6), (33, 22), (256, 256), (20, 18), (300, 136)])
def test_head_sizes(d, rot, interleaved, dt):
    say("case rotary", d, rot, interleaved, dt)
    for tokens, heads, kv in ((1, 1, 1), (7, 6, 2), (130, 3, 3)):
        Q, K, at, f = rows(tokens, heads, d, dt), rows(tokens, kv, d, dt, 2), places(tokens, 5000), sp.sp_rotary_frequencies(rot, device="cpu")
        q, k = sp.sp_rotary(at.to(DEV), f.to(DEV), Q.to(DEV), K.to(DEV), interleaved=interleaved, scale=1.25)
        close(q, *rotated(Q, at, f, interleaved, 1.25), "Q")
        close(k, *rotated(K, at, f, interleaved, 1.25), "K")
        q, k = sp.sp_rotary_grad(at.to(DEV), f.to(DEV), Q.to(DEV), K.to(DEV), interleaved=interleaved, scale=1.25)
        close(q, *rotated(Q, at, f, interleaved, 1.25, back=True), "dQ")
        close(k, *rotated(K, at, f, interleaved, 1.25, back=True), "dK")


@pytest.mark.parametrize("tokens,heads,kv,d", [(1, 32, 8, 128), (3, 64, 0, 64), (1000, 1, 1, 32), (517, 24, 24, 64), (2049, 2, 1, 128)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_tokens_and_heads(tokens, heads, kv, d, dt):
    say("case rotary", tokens, heads, kv, d, dt)
    Q, at, f = rows(tokens, heads, d, dt), places(tokens, 100000), sp.sp_rotary_frequencies(d, factor=8.0, trained=4096, device="cpu")
    if kv == 0:
        close(sp.sp_rotary(at.to(DEV), f.to(DEV), Q.to(DEV)), *rotated(Q, at, f))
        return
    K = rows(tokens, kv, d, dt, 5)
    q, k = sp.sp_rotary(at.to(DEV), f.to(DEV), Q.to(DEV), K.to(DEV))
    close(q, *rotated(Q, at, f), "Q")
    close(k, *rotated(K, at, f), "K")


def test_far_and_negative_positions():
    at = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 20, 123456789, -77], dtype=torch.int32)
    f = sp.sp_rotary_frequencies(32, device="cpu")
    for dt in (F32, BF16):
        Q = rows(8, 3, 32, dt)
        close(sp.sp_rotary(at.to(DEV), f.to(DEV), Q.to(DEV)), *rotated(Q, at, f))
    quarter = torch.tensor([torch.pi / 2, torch.pi / 4], dtype=torch.float64)   # exact quarters and eighths of a turn
    Q, at = rows(64, 1, 4, F32), torch.arange(-32, 32, dtype=torch.int32)
    close(sp.sp_rotary(at.to(DEV), quarter.to(DEV), Q.to(DEV)), *rotated(Q, at, quarter))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts(interleaved, dt):
    """Heads outside, gaps between rows, addresses that are not aligned, an input that is broadcast, in place."""
    at, f = places(40, 3000), sp.sp_rotary_frequencies(32, device="cpu")
    turn = dict(interleaved=interleaved)
    for first in (0, 1, 3):                              # the address moves by so many numbers
        whole = torch.zeros(40 * 5 * 48 + 8, dtype=dt, device=DEV)
        Q = rows(40, 5, 48, dt, first)
        view = whole[first:first + 40 * 5 * 48].view(40, 5, 48)
        view.copy_(Q)
        out = torch.full((40 * 5 * 48 + 8,), 7.0, dtype=dt, device=DEV)
        to = out[first:first + 40 * 5 * 48].view(40, 5, 48)
        assert sp.sp_rotary(at.to(DEV), f.to(DEV), view, Q_out=to, **turn) is to
        close(to, *rotated(Q, at, f, interleaved), "moved by %d" % first)
        assert (out[:first] == 7).all() and (out[first + 40 * 5 * 48:] == 7).all()
        sp.sp_rotary(at.to(DEV), f.to(DEV), view, Q_out=view, **turn)
        close(view, *rotated(Q, at, f, interleaved), "in place")
        assert (whole[:first] == 0).all() and (whole[first + 40 * 5 * 48:] == 0).all()
    Q, K = rows(40, 5, 48, dt), rows(40, 2, 48, dt, 9)
    outside = Q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)            # heads x tokens x d in memory
    both = torch.zeros(40, 7, 64, dtype=dt, device=DEV)                         # Q and K side by side, 16 numbers between heads
    q, k = sp.sp_rotary(at.to(DEV), f.to(DEV), outside, K.to(DEV), Q_out=both[:, :5, :48], K_out=both[:, 5:, :48], **turn)
    close(q, *rotated(Q, at, f, interleaved))
    close(k, *rotated(K, at, f, interleaved))
    assert (both[:, :, 48:] == 0).all()
    one = Q[:, :1].to(DEV).expand(40, 6, 48)             # one head seen as six
    close(sp.sp_rotary(at.to(DEV), f.to(DEV), one, **turn), *rotated(Q[:, :1].expand(40, 6, 48), at, f, interleaved))
    same = Q[:1].to(DEV).expand(40, 5, 48)               # one token seen as forty
    close(sp.sp_rotary_grad(at.to(DEV), f.to(DEV), same, **turn), *rotated(Q[:1].expand(40, 5, 48), at, f, interleaved, back=True))


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_pairs_at_any_number_of_elements(interleaved, dt):
    """Heads and rows an odd number of elements apart, and addresses moved by one: pairs begin anywhere; in place too."""
    say("case rotary, odd strides", interleaved, dt)
    at, f = places(29, 3000), sp.sp_rotary_frequencies(22, device="cpu")
    for first in (0, 1):
        whole = torch.full((first + 29 * 5 * 33 + 4,), 7.0, dtype=dt, device=DEV)
        view, Q = whole[first:first + 29 * 5 * 33].view(29, 5, 33), rows(29, 5, 33, dt, first)
        for grad, call in ((False, sp.sp_rotary), (True, sp.sp_rotary_grad)):
            view.copy_(Q)
            close(call(at.to(DEV), f.to(DEV), view, interleaved=interleaved), *rotated(Q, at, f, interleaved, back=grad))
            call(at.to(DEV), f.to(DEV), view, None, interleaved, 1.0, view)
            close(view, *rotated(Q, at, f, interleaved, back=grad))
            assert (whole[:first] == 7).all() and (whole[first + 29 * 5 * 33:] == 7).all()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(2048, 2048), (2050, 2050), (4100, 4096), (2307, 2306)])
def test_heads_of_more_pairs_than_are_kept(d, rot, interleaved, dt):
    """1024 pairs have room in the LDS; of more every item makes its own cosines.  Both sides of the border, both pairings, the gradient."""
    say("case rotary, many pairs", d, rot, interleaved, dt)
    Q, K, at, f = rows(37, 2, d, dt), rows(37, 1, d, dt, 2), places(37, 5000), sp.sp_rotary_frequencies(rot, device="cpu")
    for grad, call in ((False, sp.sp_rotary), (True, sp.sp_rotary_grad)):
        q, k = call(at.to(DEV), f.to(DEV), Q.to(DEV), K.to(DEV), interleaved=interleaved, scale=0.75)
        close(q, *rotated(Q, at, f, interleaved, 0.75, back=grad), "Q")
        close(k, *rotated(K, at, f, interleaved, 0.75, back=grad), "K")


def test_gradient_against_differentiation():
    """<dY, rotary(X)> differentiated by torch in 64 bits, and by differences of the kernel's own results (which are linear in X)."""
    for interleaved in (False, True):
        X, dY, at, f = rows(9, 2, 24, F32), rows(9, 2, 24, F32, 4), places(9, 500), sp.sp_rotary_frequencies(16, device="cpu")
        leaf = X.double().requires_grad_()
        a = at.double()[:, None] * f
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        p, q = (leaf[..., 0:16:2], leaf[..., 1:16:2]) if interleaved else (leaf[..., :8], leaf[..., 8:16])
        y, z = p * c - q * s, p * s + q * c
        y = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
        want, = torch.autograd.grad((torch.cat([y, leaf[..., 16:]], -1) * dY.double()).sum(), leaf)
        got = sp.sp_rotary_grad(at.to(DEV), f.to(DEV), dY.to(DEV), interleaved=interleaved)
        close(got, want, rotated(dY, at, f, interleaved, back=True)[1])
        for d in (0, 5, 15, 20):
            step = torch.zeros_like(X)
            step[:, :, d] = 1
            turned = sp.sp_rotary(at.to(DEV), f.to(DEV), step.to(DEV), interleaved=interleaved)
            by_difference = (turned.double().cpu() * dY.double()).sum(-1)
            assert (by_difference - got.double().cpu()[..., d]).abs().max() < 40 * 2.0 ** -24 * dY.abs().sum(-1).max()


def test_numbers_that_are_not_finite_stay_in_their_pair():
    Q = rows(3, 2, 16, F32)
    Q[1, 0, 3], Q[2, 1, 13] = float("nan"), float("inf")
    at, f = torch.tensor([5, 6, 7], dtype=torch.int32), sp.sp_rotary_frequencies(12, device="cpu")
    y = sp.sp_rotary(at.to(DEV), f.to(DEV), Q.to(DEV)).cpu()
    assert torch.isnan(y).nonzero().tolist() == [[1, 0, 3], [1, 0, 9]] and torch.isinf(y).nonzero().tolist() == [[2, 1, 13]]


def test_nothing_to_do():
    f = sp.sp_rotary_frequencies(16)
    assert sp.sp_rotary(torch.zeros(0, dtype=torch.int32, device=DEV), f, torch.zeros(0, 2, 16, device=DEV)).shape == (0, 2, 16)
    q, k = sp.sp_rotary(torch.zeros(3, dtype=torch.int32, device=DEV), f, torch.zeros(3, 0, 16, device=DEV), torch.ones(3, 1, 16, device=DEV))
    assert q.shape == (3, 0, 16) and (k == 1).all()


def test_refused_arguments():
    f, at, Q = sp.sp_rotary_frequencies(16), torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, 2, 16, device=DEV)
    for bad in (at.long(), at.cpu(), at[:2], torch.zeros(6, dtype=torch.int32, device=DEV)[::2]):
        with pytest.raises(ValueError):
            sp.sp_rotary(bad, f, Q)
    for bad in (f.float(), f.cpu(), f[None], f[::2]):
        with pytest.raises(ValueError):
            sp.sp_rotary(at, bad, Q)
    for K in (torch.zeros(2, 2, 16, device=DEV), torch.zeros(3, 2, 8, device=DEV), torch.zeros(3, 2, 16, device=DEV).half(), torch.zeros(3, 2, 16)):
        with pytest.raises(ValueError):
            sp.sp_rotary(at, f, Q, K)
    for out in (Q[:2], Q.half(), torch.zeros(3, 2, 32, device=DEV)[..., ::2]):
        with pytest.raises(ValueError):
            sp.sp_rotary(at, f, Q, Q_out=out)
    with pytest.raises(sp.SpError):
        sp.sp_rotary(at, f, Q.double())
    with pytest.raises(sp.SpError):
        sp.sp_rotary(at, sp.sp_rotary_frequencies(18), Q)
    with pytest.raises(sp.SpError):                      # rows that would be written over each other
        sp.sp_rotary(at, f, Q, Q_out=torch.zeros(1, 2, 16, device=DEV).expand(3, 2, 16))


def test_graphs_and_streams():
    at, f, Q, K = places(33, 900).to(DEV), sp.sp_rotary_frequencies(64), rows(33, 8, 64, BF16).to(DEV), rows(33, 2, 64, BF16, 3).to(DEV)
    qo, ko = torch.empty_like(Q), torch.empty_like(K)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sp.sp_rotary(at, f, Q, K, Q_out=qo, K_out=ko)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.sp_rotary(at, f, Q, K, Q_out=qo, K_out=ko)
    for seed in range(3):
        Q.copy_(rows(33, 8, 64, BF16, 20 + seed))
        at.copy_(places(33, 900, seed))
        graph.replay()
        q, k = sp.sp_rotary(at, f, Q, K)
        torch.cuda.synchronize()
        assert torch.equal(q, qo) and torch.equal(k, ko)
        close(qo, *rotated(Q.cpu(), at.cpu(), f.cpu()))


def test_large_offsets():
    """Rows that lie beyond 2^32 bytes."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GiB")
    whole = torch.zeros((1 << 32) + 4096, dtype=BF16, device=DEV)
    Q, at, f = rows(2, 3, 64, BF16), places(2, 100), sp.sp_rotary_frequencies(64, device="cpu")
    view = whole.as_strided((2, 3, 64), (1 << 32, 64, 1))
    view.copy_(Q)
    sp.sp_rotary(at.to(DEV), f.to(DEV), view, Q_out=view)
    close(view, *rotated(Q, at, f))
