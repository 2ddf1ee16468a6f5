"""Attention over a stored pattern, without a GPU: the binding's structures against the header, refusals that need no tensor, and the
definition in 64 bits that the GPU tests compare with, against torch's softmax and automatic differentiation."""
import ctypes
import os
import re

import pytest
import torch

import paper_2202_04305_amd as sp
from attention_util import Problem, buckets_of, reference
from paper_2202_04305_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"int": ctypes.c_int, "int64_t": ctypes.c_int64, "double": ctypes.c_double}


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


@pytest.mark.parametrize("name,mirror", [("sp_attention_problem", binding.SpAttentionProblem), ("sp_attention_grads", binding.SpAttentionGrads)])
def test_structures_match_the_header(name, mirror):
    assert fields(name) == list(mirror._fields_)


def test_null_handles_are_refused():
    L = sp.load_library()
    p, g, size = binding.SpAttentionProblem(), binding.SpAttentionGrads(), ctypes.c_size_t(7)
    assert L.sp_prepare_attention(None, 0, None) == 1
    assert L.sp_attention_workspace(None, ctypes.byref(p), 0, ctypes.byref(size)) == 1 and size.value == 0
    assert L.sp_attention_workspace(None, ctypes.byref(p), 0, None) == 1
    assert L.sp_attention(None, ctypes.byref(p), None, 0, 0, None, None, 0, None) == 1
    assert L.sp_attention(None, None, None, 0, 0, None, None, 0, None) == 1
    assert L.sp_attention_grad(None, ctypes.byref(p), ctypes.byref(g), None, 0, None) == 1
    assert L.sp_attention_grad(None, None, None, None, 0, None) == 1


def test_buckets():
    """Borders that are whole numbers are taken exactly: 8 exact distances, then 8 far buckets up to 128, one for each half power of two."""
    d = torch.arange(0, 400)
    b = buckets_of(-d, 16, 128, False)
    assert b[:8].tolist() == list(range(8))
    for k in range(8):
        first = int((b == 8 + k).nonzero()[0])
        assert first == -int(-8 * 2 ** (k / 2) // 1) if k % 2 else first == 8 * 2 ** (k // 2)
    assert int(b[-1]) == 15
    both = buckets_of(torch.tensor([-200, -1, 0, 1, 200]), 32, 128, True)
    assert both.tolist() == [15, 1, 0, 17, 31]


@pytest.mark.parametrize("causal,buckets", [(False, 0), (False, 8), (True, 8), (True, 0)])
def test_reference_against_automatic_differentiation(causal, buckets):
    g = torch.Generator().manual_seed(1)
    m, n, H, Hk, D = 13, 17, 6, 2, 5
    at = torch.rand(m, n, generator=g) < 0.6
    at[4] = False
    Q, K, V = (torch.randn(s, generator=g).double() for s in ((m, H, D), (n, Hk, D), (n, Hk, D)))
    dO = torch.randn(m, H, D, generator=g).double()
    pos = torch.arange(m, dtype=torch.int32), torch.arange(n, dtype=torch.int32) - 2
    p = Problem(at, Q.float(), K.float(), V.float(), causal=causal, qpos=pos[0], kpos=pos[1], max_distance=9, dO=dO.float())
    if buckets:
        p.bias = torch.randn(buckets, H, generator=g)
    leaves = [t.double().requires_grad_() for t in (p.Q, p.K, p.V)] + ([p.bias.double().requires_grad_()] if buckets else [])
    s = torch.einsum("ihd,jhd->hij", leaves[0], leaves[1].repeat_interleave(H // Hk, 1)) * p.scale
    rel = pos[1].long()[None, :] - pos[0].long()[:, None]
    if buckets:
        s = s + leaves[3][buckets_of(rel, buckets, 9, True)].permute(2, 0, 1)
    keep = at & (rel <= 0) if causal else at
    some = keep.any(1)
    w = torch.softmax(s.masked_fill(~keep, float("-inf"))[:, some], -1)
    O = torch.zeros(m, H, D, dtype=torch.float64)
    O[some] = torch.einsum("hij,jhd->ihd", w, leaves[2].repeat_interleave(H // Hk, 1))
    grads = torch.autograd.grad((O * p.dO.double()).sum(), leaves)
    ref = reference(p)
    assert torch.allclose(ref["O"][0], O.detach(), atol=1e-12)
    for k, t in zip(("dQ", "dK", "dV", "dT"), grads):
        assert torch.allclose(ref[k][0], t, atol=1e-11), k
    assert all(bool((tol >= 0).all()) and bool(torch.isfinite(tol).all()) for _, tol in ref.values())
