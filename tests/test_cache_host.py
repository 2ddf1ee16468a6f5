"""The cache held in 4 bits and rotary positions, without a GPU: the binding's structures against the header, every refusal (they come before
anything is launched), frequencies, and the definitions that the GPU tests compare with."""
import contextlib
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

import paper_2202_04305_amd as sp
import cache_util as U
from paper_2202_04305_amd import binding as B
from paper_2202_04305_amd import build
from test_device_assembly import OBJDUMP, lost_registers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"int": ctypes.c_int, "int64_t": ctypes.c_int64, "double": ctypes.c_double}
NULL, SHAPE, DTYPE, UNSUPPORTED, TOO_LARGE = 1, 8, 9, 10, 11
SOME = 1 << 20                           # an address that nothing may look at: every call here is refused


def fields(name):
    text = open(os.path.join(ROOT, "include", "spmi.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    out = []
    for decl in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";"):
        if decl.strip():
            kind, names = re.match(r"\s*(?:const\s+)?(\w+)\s+(.*)", decl, flags=re.S).groups()
            for n in names.split(","):
                out.append((n.strip().lstrip("*"), ctypes.c_void_p if n.strip().startswith("*") else TYPES[kind]))
    return out


@pytest.mark.parametrize("name,mirror", [("sp_rotary_problem", B.SpRotaryProblem), ("sp_cache", B.SpCache), ("sp_cache_step", B.SpCacheStep),
                                         ("sp_cache_problem", B.SpCacheProblem)])
def test_structures_match_the_header(name, mirror):
    assert fields(name) == list(mirror._fields_)


@pytest.mark.parametrize("pack,mirror", [(B._ROTARY, B.SpRotaryProblem), (B._STEP, B.SpCacheStep), (B._PROBLEM, B.SpCacheProblem)])
def test_packed_bytes_are_the_structures(pack, mirror):
    """The binding packs the bytes of these structures: the same ones, field by field (padding aside, which both leave zero)."""
    numbers = [k + 1 for k in range(len(mirror._fields_))]
    assert pack.size == ctypes.sizeof(mirror) and pack.pack(*numbers) == bytes(mirror(*numbers))


def ref(s):
    return ctypes.byref(s)


def cache(**more):
    return B.SpCache(**{**dict(data=SOME, pages=10, pageTokens=16, kvHeads=2, headDim=64), **more})


BAD_CACHES = [(dict(pages=-1), SHAPE), (dict(pageTokens=0), SHAPE), (dict(pageTokens=24), SHAPE), (dict(pageTokens=-16), SHAPE), (dict(kvHeads=0), SHAPE),
              (dict(kvHeads=65536), SHAPE), (dict(headDim=0), SHAPE), (dict(headDim=257), SHAPE), (dict(pages=1 << 27), TOO_LARGE),
              (dict(pages=1 << 62), TOO_LARGE)]


class _OnGpu3:
    """What the entry points ask of a tensor before they make its device current."""
    dtype, _index = torch.int32, 3

    def get_device(self):
        return 3


@pytest.mark.parametrize("call", [
    lambda t: sp.sp_rotary(t, t, t), lambda t: sp.sp_rotary_grad(t, t, t), lambda t: sp.sp_cache_map(t, t, t, t, t, 16, 4, 5), lambda t: sp.sp_cache_store(t, t, t, t),
    lambda t: sp.sp_cache_load(t, t), lambda t: sp.sp_cache_attention(t, t, t, t, t)])
def test_entry_points_make_the_tensors_device_current(call, monkeypatch):
    """Without a GPU: torch's device functions are stood in for; whatever the call does first is done with the tensors' device current."""
    now, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d
        yield
        now[0] = before

    def inner(*args, **more):
        seen.append(now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    for name in ("_rotary", "_cache_map", "_cache_store", "_cache_load", "_cache_attention"):
        monkeypatch.setattr(B, name, inner)
    call(_OnGpu3())
    assert seen == [3] and now == [0]


def test_cache_bytes():
    L, size = sp.load_library(), ctypes.c_size_t(7)
    for d, row in ((1, 17), (32, 17), (33, 34), (64, 34), (65, 52), (96, 52), (97, 68), (128, 68), (129, 88), (160, 88), (192, 104), (256, 136)):
        assert L.sp_cache_bytes(ref(cache(headDim=d, pages=3, pageTokens=48, kvHeads=5)), ref(size)) == 0
        assert size.value == 3 * 48 * 5 * 2 * row, d
    assert L.sp_cache_bytes(ref(cache(pages=0)), ref(size)) == 0 and size.value == 0
    assert L.sp_cache_bytes(ref(cache(pages=(1 << 27) - 1)), ref(size)) == 0
    for more, code in BAD_CACHES:
        assert L.sp_cache_bytes(ref(cache(**more)), ref(size)) == code and size.value == 0, more
    assert L.sp_cache_bytes(None, ref(size)) == NULL and L.sp_cache_bytes(ref(cache()), None) == NULL


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), "meta"])
def test_a_cache_is_on_a_gpu(device):
    """Kernels would be given the address of memory that they cannot read: no such cache is made, nor any of its tensors looked at."""
    with pytest.raises(ValueError):
        sp.sp_cache(4, 16, 2, 64, device=device)
    with pytest.raises(ValueError):
        sp.Cache(torch.zeros(1 << 16, dtype=torch.uint8, device=device), cache())


def rotary(**more):
    return B.SpRotaryProblem(**{**dict(dtype=3, headDim=64, rotDim=32, interleaved=0, scale=1.0, tokens=5, position=SOME, frequency=SOME, heads=4, kvHeads=2,
                                       Q=SOME, ldq=256, hdq=64, K=SOME, ldk=128, hdk=64, Qout=SOME, ldqo=256, hdqo=64, Kout=SOME, ldko=128, hdko=64), **more})


@pytest.mark.parametrize("more,code", [
    (dict(dtype=1), DTYPE), (dict(dtype=-1), DTYPE), (dict(dtype=7), DTYPE), (dict(headDim=0), SHAPE), (dict(rotDim=31), SHAPE), (dict(rotDim=66), SHAPE), (dict(rotDim=-2), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(heads=-1), SHAPE), (dict(kvHeads=-1), SHAPE), (dict(scale=math.inf), SHAPE), (dict(scale=1e300), SHAPE),
    (dict(scale=math.nan), SHAPE), (dict(ldq=-1), SHAPE), (dict(hdk=-1), SHAPE), (dict(ldqo=63), SHAPE), (dict(hdqo=63), SHAPE), (dict(ldko=63), SHAPE), (dict(hdko=63), SHAPE),
    (dict(interleaved=2), UNSUPPORTED), (dict(position=None), NULL), (dict(frequency=None), NULL), (dict(Q=None), NULL), (dict(K=None), NULL),
    (dict(Qout=None), NULL), (dict(Kout=None), NULL), (dict(dtype=1, headDim=0, interleaved=2, Q=None), DTYPE), (dict(headDim=0, interleaved=2, Q=None), SHAPE),
    (dict(interleaved=2, Q=None), UNSUPPORTED), (dict(heads=1 << 25), TOO_LARGE), (dict(heads=(1 << 31) - 1, kvHeads=(1 << 31) - 1), TOO_LARGE)])
def test_rotary_refusals(more, code):
    L = sp.load_library()
    assert L.sp_rotary(ref(rotary(**more)), None) == code
    assert L.sp_rotary_grad(ref(rotary(**more)), None) == code


def test_rotary_of_nothing():
    L = sp.load_library()
    assert L.sp_rotary(None, None) == NULL and L.sp_rotary_grad(None, None) == NULL
    for more in (dict(tokens=0, Q=None, K=None, Qout=None, Kout=None, position=None), dict(heads=0, kvHeads=0, Q=None, K=None)):
        assert L.sp_rotary(ref(rotary(**more)), None) == 0


def test_frequencies():
    f = sp.sp_rotary_frequencies(64, 10000.0, device="cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, 10000.0 ** (-torch.arange(0, 64, 2).double() / 64), rtol=1e-15)
    assert torch.equal(sp.sp_rotary_frequencies(64, 10000.0, factor=4.0, device="cpu"), f / 4)
    g = sp.sp_rotary_frequencies(64, 10000.0, factor=4.0, trained=4096, low=1.0, high=32.0, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns > 32], f[turns > 32]) and torch.equal(g[turns < 1], f[turns < 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert int(between.sum()) > 3
    c = (turns - 1) / 31
    assert torch.allclose(g[between], ((1 - c) / 4 * f + c * f)[between], rtol=1e-14)
    assert sp.sp_rotary_frequencies(0, device="cpu").numel() == 0
    L, out = sp.load_library(), (ctypes.c_double * 8)()
    for args in ((7, 1e4, 1.0, 0, 1.0, 32.0), (-2, 1e4, 1.0, 0, 1.0, 32.0), (16, 0.0, 1.0, 0, 1.0, 32.0), (16, math.nan, 1.0, 0, 1.0, 32.0), (16, math.inf, 1.0, 0, 1.0, 32.0),
                 (16, 1e4, 0.0, 0, 1.0, 32.0), (16, 1e4, math.inf, 0, 1.0, 32.0), (16, 1e4, 1.0, -1, 1.0, 32.0), (16, 1e4, 1.0, 9, 32.0, 32.0), (16, 1e4, 1.0, 9, 1.0, math.nan)):
        assert L.sp_rotary_frequencies(*args, out) == SHAPE, args
    assert L.sp_rotary_frequencies(16, 1e4, 1.0, 0, 1.0, 32.0, None) == NULL
    assert L.sp_rotary_frequencies(16, 1e4, 1.0, 0, 5.0, 5.0, out) == 0          # the borders play no part then


def test_frequencies_are_finite():
    """Borders, bases and factors that would give NaN or infinity are refused, those that give numbers are not."""
    L, out = sp.load_library(), (ctypes.c_double * 32)()
    # the least base is 2^-1074: its power -2k / rotDim is at most 2^939.75 for 16 numbers, and past 2^1024 from k = 31 of 64 on
    for args in ((16, 1e4, 1.0, 9, -math.inf, 32.0), (16, 1e4, 1.0, 9, -math.inf, math.inf), (64, 5e-324, 1.0, 0, 1.0, 32.0), (16, 1e4, 1e-310, 0, 1.0, 32.0)):
        assert L.sp_rotary_frequencies(*args, out) == SHAPE, args
        with pytest.raises(sp.SpError):
            sp.sp_rotary_frequencies(*args, device="cpu")
    for args in ((16, 1e4, 2.0, 9, 1.0, math.inf), (16, 5e-324, 1.0, 0, 1.0, 32.0), (16, 1e-300, 1.0, 0, 1.0, 32.0), (16, 1e4, 1e308, 0, -math.inf, 32.0)):
        assert L.sp_rotary_frequencies(*args, out) == 0 and all(math.isfinite(x) for x in out[:8]), args


def step(**more):
    return B.SpCacheStep(**{**dict(requests=3, tokens=5, pages=10, pageTokens=16, length=SOME, added=SOME, freePages=SOME, freeCount=4, taken=SOME, table=SOME, ldt=4,
                                   width=4, lengthOut=SOME, start=SOME, position=SOME, slot=SOME, takenOut=SOME), **more})


@pytest.mark.parametrize("more,code", [
    (dict(requests=-1), SHAPE), (dict(tokens=-1), SHAPE), (dict(pages=-1), SHAPE), (dict(freeCount=-1), SHAPE), (dict(width=-1), SHAPE), (dict(ldt=3), SHAPE),
    (dict(pageTokens=0), SHAPE), (dict(pageTokens=20), SHAPE), (dict(pages=1 << 27), TOO_LARGE), (dict(requests=1 << 31), TOO_LARGE), (dict(tokens=1 << 31), TOO_LARGE),
    *[({k: None}, NULL) for k in ("length", "added", "freePages", "taken", "table", "lengthOut", "start", "position", "slot", "takenOut")],
    (dict(pages=1 << 27, ldt=3), SHAPE), (dict(pages=1 << 27, taken=None), TOO_LARGE)])
def test_map_refusals(more, code):
    assert sp.load_library().sp_cache_map(ref(step(**more)), None) == code
    assert sp.load_library().sp_cache_map(None, None) == NULL


def test_store_and_load_refusals():
    L = sp.load_library()

    def both(c, dtype=3, tokens=5, slot=SOME, K=SOME, ldk=128, hdk=64, V=SOME, ldv=128, hdv=64):
        return [f(c if c is None else ref(c), dtype, tokens, slot, K, ldk, hdk, V, ldv, hdv, None) for f in (L.sp_cache_store, L.sp_cache_load)]
    assert both(None) == [NULL, NULL]
    for dtype in (1, -1, 9):
        assert both(cache(), dtype=dtype) == [DTYPE, DTYPE]
    for more, code in BAD_CACHES:
        assert both(cache(**more)) == [code, code]
    for more in (dict(tokens=-1), dict(ldk=-1), dict(hdk=-1), dict(ldv=-1), dict(hdv=-1)):
        assert both(cache(), **more) == [SHAPE, SHAPE]
    for more in (dict(ldk=63), dict(hdk=63), dict(ldv=63), dict(hdv=63)):      # rows that would be written over each other
        assert both(cache(), **more)[1] == SHAPE
    assert both(cache(), tokens=1 << 31) == [TOO_LARGE, TOO_LARGE]
    for more in (dict(slot=None), dict(K=None), dict(V=None)):
        assert both(cache(), **more) == [NULL, NULL]
    assert both(cache(data=None)) == [NULL, NULL]
    assert both(cache(data=None), tokens=0, slot=None, K=None, V=None) == [0, 0]
    assert both(cache(pages=0, data=None))[0] == 0                             # nowhere to store to


def test_limits_of_a_launch():
    """Both sides of what the header says: 2^24 workgroups of 32 rows and one head, or of 64 requests.  (A cache without pages: nothing is launched.)"""
    L = sp.load_library()
    for heads, tokens in ((1 << 15, 511 * 32), (1, (1 << 29) - 32), (65535, 256 * 32), (8192, 2047 * 32)):
        row = (SOME, heads * 64, 64, SOME, heads * 64, 64, None)
        wide = cache(kvHeads=heads, pages=0)
        assert L.sp_cache_store(ref(wide), 3, tokens, SOME, *row) == 0, (heads, tokens)
        assert L.sp_cache_store(ref(wide), 3, tokens + 1, SOME, *row) == TOO_LARGE and L.sp_cache_load(ref(wide), 3, tokens + 1, SOME, *row) == TOO_LARGE, (heads, tokens)
    assert L.sp_cache_map(ref(step(requests=(1 << 30) - 63)), None) == TOO_LARGE


def problem(**more):
    return B.SpCacheProblem(**{**dict(dtype=3, heads=4, causal=1, scale=0.1, requests=3, tokens=5, Q=SOME, ldq=256, hdq=64, table=SOME, ldt=4, width=4, length=SOME,
                                      start=SOME), **more})


@pytest.mark.parametrize("more,code", [
    (dict(dtype=1), DTYPE), (dict(dtype=5), DTYPE), (dict(heads=0), SHAPE), (dict(heads=3), SHAPE), (dict(heads=65536), SHAPE), (dict(requests=-1), SHAPE), (dict(tokens=-1), SHAPE),
    (dict(width=-1), SHAPE), (dict(ldt=3), SHAPE), (dict(ldq=-1), SHAPE), (dict(hdq=-1), SHAPE), (dict(scale=math.nan), SHAPE), (dict(scale=3e38), SHAPE),
    (dict(causal=2), UNSUPPORTED), (dict(causal=-1), UNSUPPORTED), (dict(requests=1 << 31), TOO_LARGE), (dict(tokens=1 << 31), TOO_LARGE),
    (dict(tokens=(1 << 31) - 1, heads=65534), TOO_LARGE)])
def test_attention_refusals(more, code):
    L, size = sp.load_library(), ctypes.c_size_t(7)
    assert L.sp_cache_attention(ref(cache()), ref(problem(**more)), SOME, 256, 64, None, SOME, 1 << 40, None) == code
    assert L.sp_cache_attention_workspace(ref(cache()), ref(problem(**more)), ref(size)) == code and size.value == 0


def test_more_attention_refusals():
    L, size = sp.load_library(), ctypes.c_size_t(7)

    def call(c=cache(), p=problem(), O=SOME, ldo=256, hdo=64, work=SOME, room=1 << 40):
        return L.sp_cache_attention(c if c is None else ref(c), p if p is None else ref(p), O, ldo, hdo, None, work, room, None)
    assert call(c=None) == NULL and call(p=None) == NULL
    for more, code in BAD_CACHES:
        assert call(c=cache(**more)) == code
    assert call(ldo=63) == SHAPE and call(hdo=63) == SHAPE
    assert call(O=None) == NULL and call(c=cache(data=None)) == NULL
    for k in ("Q", "table", "length", "start"):
        assert call(p=problem(**{k: None})) == NULL, k
    assert call(p=problem(tokens=0, Q=None), O=None, work=None, room=0) == 0
    assert call(p=problem(requests=0, length=None, table=None), O=None, work=None, room=0) == 0
    assert L.sp_cache_attention_workspace(None, ref(problem()), ref(size)) == NULL and size.value == 0
    assert L.sp_cache_attention_workspace(ref(cache()), None, ref(size)) == NULL
    assert L.sp_cache_attention_workspace(ref(cache()), ref(problem()), None) == NULL
    # a workspace that is missing, too small or not aligned, where one is needed
    large = problem(requests=1, width=100000, ldt=100000)
    assert L.sp_cache_attention_workspace(ref(cache(pages=100000)), ref(large), ref(size)) == 0
    if size.value:
        assert call(c=cache(pages=100000), p=large, work=None) == NULL
        assert call(c=cache(pages=100000), p=large, room=size.value - 1) == SHAPE
        assert call(c=cache(pages=100000), p=large, work=SOME + 128) == SHAPE


def test_what_is_held():
    """The definition against numbers worked out by hand."""
    x = torch.tensor([[7.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.01, -0.0, 6.9], [7.001, 0.5, 0.51, 1.5, 2.5, 3.5, 5.0, 7.0, -7.0, 1.0, 2.0, 0.0]])
    assert U.held(x).tolist() == [[6, 0, 0.5, 1, 1, 2, 2, 4, 4, -6, 0, 6], [8, 0, 1, 2, 2, 4, 4, 8, -8, 1, 2, 0]]
    y = torch.randn(50, 3, 70) * torch.exp2(torch.randint(-30, 30, (50, 3, 1)).float())
    assert torch.equal(U.held(U.held(y)), U.held(y))                           # what is held stays as it is when stored again
    assert torch.equal(U.held(y).bfloat16().double(), U.held(y))
    z = torch.zeros(2, 64)
    z[0, 3], z[1, 40] = float("inf"), float("nan")
    assert torch.isnan(U.held(z)).sum(-1).tolist() == [32, 32] and torch.isnan(U.held(z)[0, :32]).all()
    big = torch.tensor([[3.4e38, 1e38, 1.0], [1e-44, 1e-30, 0.0]])
    assert U.held(big)[0].tolist() == [6 * 2.0 ** 125, 2 * 2.0 ** 125, 0.0] and U.held(big)[1, 0] == 0


def test_reference_attention():
    """The reference against torch's softmax, pages out of order."""
    torch.manual_seed(3)
    P, pages, G, H, D = 16, 9, 2, 6, 5
    K, V = torch.randn(pages * P, G, D).double(), torch.randn(pages * P, G, D).double()
    table = torch.tensor([[4, 2, 7], [1, -1, 0], [8, 3, 5]], dtype=torch.int32)
    lengths, start = [37, 48, 0], [0, 3, 4, 6]
    Q = torch.randn(7, H, D)
    got = U.attended(K, V, Q, table, lengths, start, P, pages)
    slots = [[4 * P + t for t in range(16)] + [2 * P + t for t in range(16)] + [7 * P + t for t in range(5)], [P + t for t in range(16)] + list(range(16))]
    for row, upto in ((0, 35), (1, 36), (2, 37), (3, 32)):
        for h in range(H):
            j = slots[0 if row < 3 else 1][:upto]
            s = K[j, h // 3] @ Q[row, h].double() * D ** -0.5
            assert torch.allclose(got["O"][0][row, h], torch.softmax(s, 0) @ V[j, h // 3], atol=1e-12)
            assert abs(got["lse"][0][h, row] - torch.logsumexp(s, 0)) < 1e-12
    assert (got["O"][0][4:6] == 0).all() and (got["lse"][0][:, 4:6] == float("-inf")).all() and torch.isnan(got["O"][0][6]).all()
    assert all(bool((tol[:6] if k == "O" else tol[:, :6]).isfinite().all()) for k, (_, tol) in got.items())


def test_no_kernel_of_the_cache_loses_what_it_keeps_aside(tmp_path):
    """As for the kernels of attention over a pattern: what the compiler keeps in accumulation registers or scratch is fetched again, all of it."""
    lib = tmp_path / "lib.so"
    build.is_stale() and build.build()
    lib.write_bytes(open(build.LIB, "rb").read())
    subprocess.check_call([OBJDUMP, "--offloading", str(lib)], stdout=subprocess.DEVNULL, cwd=tmp_path)
    kernels = 0
    for part in sorted(tmp_path.glob("lib.so.*gfx950")):
        names = subprocess.run([OBJDUMP, "-t", str(part)], stdout=subprocess.PIPE, text=True, check=True).stdout
        if not re.search(r"cache_(few|many|join)_kernel", names):
            continue
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(part)], stdout=subprocess.PIPE, text=True, check=True).stdout.splitlines()
        kernels += sum(bool(re.match(r"[0-9a-f]+ <\S*cache_(few|many|join)_kernel", l)) for l in asm)
        assert lost_registers(asm) == {}
    assert kernels == 3 * 8 * 3, kernels


CHUNKS = r"""
#include "cache_attention.h"
#include <stdio.h>
#include <stdlib.h>
// argv: heads of the cache, quarters of growth, then tiles and tokens of requests.  Prints the chunks' length and every request's counts.
int main(int argc, char **argv)
{
    cache_attn_args a = {};
    a.c.G = atoi(argv[1]);
    uint64_t work = 0;
    for (int k = 3; k < argc; k += 2) work += strtoull(argv[k], 0, 10) * strtoull(argv[k + 1], 0, 10);
    const uint32_t length = cache_grown(cache_chunk_tokens(a, work), atoi(argv[2]));
    printf("%u %lld\n", length, (long long)cache_slots(a.c.G));
    for (int k = 3; k < argc; k += 2) {
        cache_request q = {};
        q.tiles = (uint32_t)strtoul(argv[k], 0, 10); q.tokens = (uint32_t)strtoul(argv[k + 1], 0, 10);
        const cache_counts c = cache_counts_of(q, length);
        printf("%u %u %u %u\n", c.chunks, c.items, c.slots, c.joins);
    }
}
"""


@pytest.fixture(scope="module")
def chunks(tmp_path_factory):
    """The attention's own arithmetic of chunks, as a program of the host."""
    d = tmp_path_factory.mktemp("chunks")
    (d / "chunks.hip").write_text(CHUNKS)
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-O1", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(os.path.dirname(build.LIB), "csrc"), "-o", str(d / "chunks"), str(d / "chunks.hip")],
                          stderr=subprocess.DEVNULL)

    def run(*numbers):
        out = subprocess.run([str(d / "chunks")] + [str(x) for x in numbers], stdout=subprocess.PIPE, text=True, check=True).stdout.split()
        return int(out[0]), int(out[1]), [tuple(map(int, out[k:k + 4])) for k in range(2, len(out), 4)]
    return run


@pytest.mark.parametrize("requests", [[(1, 2000)], [(128, 2 ** 31 - 1)], [(1, 2 ** 31 - 1)] * 3, [(5000, 2 ** 31 - 1), (1, 1)], [(3, 2 ** 31 - 256), (70, 2 ** 31 - 255)],
                                      [(300, 8000), (1, 1 << 20), (1, 0), (7, 300)], [(1 << 20, 2 ** 31 - 1)], [(40, 2 ** 31 - 1)] * 2])
@pytest.mark.parametrize("G", [1, 8, 100, 512, 65535])
def test_chunks_have_room(requests, G, chunks):
    """The workspace has a slot for every chunk of a request that is cut, and chunks cover their request, up to the longest that there may be."""
    for times in range(5):
        length, room, counts = chunks(G, times, *[x for r in requests for x in r])
        assert 256 <= length <= 1 << 31 and length % 64 == 0
        assert sum(c[2] for c in counts) < room or not any(c[2] for c in counts), (times, length, counts)
        for (tiles, tokens), (n, items, slots, joins) in zip(requests, counts):
            assert n == max(1, -(-tokens // length)) and items == tiles * n and (slots, joins) == ((items, tiles) if n > 1 else (0, 0))
