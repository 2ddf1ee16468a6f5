"""The 4-bit cache, rotary positions and attention over pages, from their definitions in 64 bits on the CPU, with the error that the GPU's
arithmetic may have.

The bounds count roundings.  u = half a step of the operands' type (eps / 2), v = 2^-24 (f32, in which everything is summed):
  a score s:       Q is exact, in `parts` = 1 (bf16), 2 (f16), 3 (f32) parts of bf16, so (parts D + 8) v of scale * sum |q||k|, and 4 v |s|
  a weight p:      twice the largest score error among the row's tokens above e^-200 (its own and the sum's), the sum's (tokens + 8) v, 4 v
                   for the exponential, |lse| v
  p as an operand: u more
  a result O:      u of itself, and (parts tokens + 8) v of the sum of the absolute terms; and 2^-126 of sum |V|: f32 has no normal number
                   below that, so a weight (relative to the row's largest, whose own is 1 in a total of at least 1) may be lost there
"""
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
PARTS = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}


def held(x):
    """What the cache holds of rows (.., d), in 64 bits."""
    out = torch.empty(x.shape, dtype=torch.float64)
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    for a in range(0, x.shape[-1], 32):
        b = x[..., a:a + 32].double()
        fine = torch.isfinite(b).all(-1, keepdim=True)
        top = torch.where(fine, b.abs().amax(-1, keepdim=True), torch.zeros(()).double())
        e = torch.full_like(top, -100.0)
        for k in range(-99, 126):                        # the least e with top <= 7 * 2^e
            e = torch.where(top > 7 * 2.0 ** (k - 1), float(k), e)
        y = b.abs() / torch.exp2(e)
        off = (y[..., None] - levels).abs()
        near = off.amin(-1, keepdim=True)
        even = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])    # of two as near the even one
        pick = even[(off[..., even] == near).double().argmax(-1)]
        value = torch.copysign(levels[pick] * torch.exp2(e), b)
        out[..., a:a + 32] = torch.where(fine.expand_as(b), value, torch.full_like(b, float("nan")))
    return out


def rotated(x, position, frequencies, interleaved=False, scale=1.0, back=False):
    """(value, bound) of rows (tokens, heads, d) turned by position * frequencies."""
    u, v = torch.finfo(x.dtype).eps / 2, 2.0 ** -24
    half = frequencies.numel()
    a = position.double()[:, None] * frequencies.double()
    c, s = torch.cos(a)[:, None] * scale, torch.sin(a)[:, None] * scale * (-1 if back else 1)
    y, tol = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    p, q = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = p * c - q * s, p * s + q * c
    # the cosine and sine: the angle's rounding (pi / 4 v), 4 v of their own and v for the scale; two products and a sum; the angle's 64 bits
    each = ((p.abs() + q.abs()) * abs(scale)) * (9 * v + a.abs()[:, None] * 2.0 ** -51)
    least = torch.finfo(x.dtype).tiny * torch.finfo(x.dtype).eps
    tol[..., first], tol[..., second] = each + u * (y[..., first].abs() + each) + least, each + u * (y[..., second].abs() + each) + least
    return y, tol


def mapped(lengths, added, free, taken, table, P, pages, tokens):
    """sp_cache_map by hand: lists in, a dict of int32 tensors out."""
    table = table.clone()
    R, width = table.shape
    start, position, slot, after = [0], [], [], []
    for r in range(R):
        have, add = max(0, lengths[r]), max(0, added[r])
        for j in range(-(-have // P), -(-(have + add) // P)):
            page = free[taken] if 0 <= taken < len(free) else -1
            taken += 1
            if j < width:
                table[r, j] = page if 0 <= page < pages else -1
        for t in range(have, have + add):
            page = int(table[r, t // P]) if t // P < width else -1
            position.append(t)
            slot.append(page * P + t % P if 0 <= page < pages else -1)
        start.append(start[-1] + add)
        after.append(have + add)
    position, slot = ([*x, *[-1] * tokens][:tokens] for x in (position, slot))
    return {k: torch.tensor(x, dtype=torch.int32) for k, x in
            (("lengths", after), ("start", start), ("position", position), ("slot", slot), ("taken", [taken]))} | {"table": table}


def attended(K, V, Q, table, lengths, start, P, pages, scale=None, causal=True):
    """{name: (value, bound)} of attention over pages whose slots hold K and V (slots, kv heads, d) in 64 bits; rows of no request: NaN."""
    m, H, D = Q.shape
    G = K.shape[1]
    scale = D ** -0.5 if scale is None else scale
    u, v, parts = torch.finfo(Q.dtype).eps / 2, 2.0 ** -24, PARTS[Q.dtype]
    least = torch.finfo(Q.dtype).tiny * torch.finfo(Q.dtype).eps
    O, O_tol = (torch.full((m, H, D), float("nan"), dtype=torch.float64) for _ in range(2))
    L, L_tol = (torch.full((H, m), float("nan"), dtype=torch.float64) for _ in range(2))
    q64 = Q.double()
    for r in range(len(lengths)):
        a, b, length = start[r], start[r + 1], lengths[r]
        if a == b:
            continue
        t = torch.arange(max(0, min(length, table.shape[1] * P)))
        page = table[r][t // P].long()
        there = (page >= 0) & (page < pages)
        t, slot = t[there], (page * P + t % P)[there]
        last = length - (b - a) + torch.arange(b - a)
        keep = (t[None] <= last[:, None]) if causal else torch.ones(b - a, t.numel(), dtype=torch.bool)
        n = keep.sum(1, keepdim=True).double()
        for h in range(H):
            k, w = K[slot, h // (H // G)], V[slot, h // (H // G)]
            s = torch.where(keep, (q64[a:b, h] @ k.T) * scale, float("-inf"))
            s = torch.where(keep & (s == float("inf")), float("nan"), s)
            top = torch.where(torch.isnan(s), float("-inf"), s).amax(1, keepdim=True) if t.numel() else torch.full((b - a, 1), float("-inf")).double()
            top = torch.where(top == float("-inf"), 0.0, top)
            e = torch.exp(s - top)
            total = e.sum(1, keepdim=True)
            none = total == 0
            lse = torch.where(none, float("-inf"), top + torch.log(total))
            p = e / torch.where(none, 1.0, total)
            # what a row does not attend to has no part in it, whatever it holds
            blank = torch.zeros((), dtype=torch.float64)
            O[a:b, h] = torch.stack([p[i, keep[i]] @ w[keep[i]] if keep[i].any() else blank.expand(D) for i in range(b - a)])
            es = (parts * D + 8) * v * abs(scale) * (q64[a:b, h].abs() @ k.abs().T) + 4 * v * s.abs()
            es = torch.where(keep & (s > lse - 200), es, 0.0)
            worst = es.amax(1, keepdim=True) if t.numel() else torch.zeros(b - a, 1).double()
            rel = 2 * worst + (n + 12) * v + v * torch.where(none, 0.0, lse).abs()
            big = torch.stack([p[i, keep[i]] @ w[keep[i]].abs() if keep[i].any() else blank.expand(D) for i in range(b - a)])
            lost = torch.stack([w[keep[i]].abs().sum(0) for i in range(b - a)]) * 2.0 ** -126
            O_tol[a:b, h] = u * O[a:b, h].abs() * (1 + rel) + big * (rel + u + (parts * n + 8) * v) + lost + least
            L[h, a:b] = lse[:, 0]
            L_tol[h, a:b] = (worst + (n + 12) * v + 3 * v * torch.where(none, 0.0, lse).abs())[:, 0]
    return {"O": (O, O_tol), "lse": (L, L_tol)}
