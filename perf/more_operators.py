"""Serving from a cache of keys and values held in 4 bits, as measurable cases: the pages and slots of a step from the requests' lengths,
rotary positions (with their gradient), keys and values into the pages and back, and attention of single tokens and of prompts over
the pages.

A case is a dict of plain values.  `op` says the operator; `lens` seeds the lengths of the requests, so that the work of a case does
not depend on the seed of its inputs.  Four bits: blocks of 32 numbers share a power of two 2^e, the least that leaves the largest of them
at 7 or below; a number is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e, with a sign (nearest, ties to the even one of their order, at most 6).
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32                  # numbers that share a scale
EXP_MIN, EXP_MAX = -100, 125


def listed():
    return [
        # one step of eight short conversations, a token each: a launch and the call are all there is
        {"name": "map_step_small", "op": "map", "requests": 8, "len": 200, "len_min": 1, "add": 1, "add_min": 1, "page": 16, "lens": 1},
        # a step that takes in many prompts beside running requests, some of which wait: pages of 64
        {"name": "map_prompts", "op": "map", "requests": 509, "len": 4096, "len_min": 0, "add": 1000, "add_min": 0, "page": 64, "lens": 2},
        # queries and keys of one step of a small batch
        {"name": "rotary_step_small", "op": "rotary", "dtype": "bf16", "tokens": 8, "heads": 32, "kv": 8, "dim": 128, "rot": 128,
         "interleaved": False, "positions": 4096, "factor": 1.0, "trained": 0, "train": False},
        # the prompts of a batch, neighbouring numbers paired, frequencies scaled for contexts far beyond the trained one
        {"name": "rotary_prompt_long", "op": "rotary", "dtype": "bf16", "tokens": 16384, "heads": 32, "kv": 8, "dim": 128, "rot": 128,
         "interleaved": True, "positions": 1048576, "factor": 16.0, "trained": 8192, "train": False},
        # a training step in single precision: a quarter of the head, odd sizes, forward and gradient
        {"name": "rotary_train_f32", "op": "rotary", "dtype": "f32", "tokens": 4099, "heads": 12, "kv": 12, "dim": 80, "rot": 20,
         "interleaved": False, "positions": 4099, "factor": 1.0, "trained": 0, "train": True},
        # one token of each of 64 requests into the pages, and read back
        {"name": "store_step", "op": "store", "dtype": "bf16", "tokens": 64, "kv": 8, "dim": 128, "page": 64, "run": 1, "lens": 3},
        # prompts into the pages, in stretches of a request each, and read back
        {"name": "store_prompts", "op": "store", "dtype": "bf16", "tokens": 32768, "kv": 8, "dim": 128, "page": 64, "run": 700, "lens": 4},
        # one step of four short conversations: launches and host work are all there is
        {"name": "attend_step_small", "op": "attend", "dtype": "bf16", "heads": 8, "kv": 8, "dim": 64, "page": 16, "requests": 4,
         "len": 200, "len_min": 64, "add": 1, "add_min": 1, "lens": 5},
        # one step of a serving batch of ragged requests
        {"name": "attend_step_batch", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 8, "dim": 128, "page": 64, "requests": 64,
         "len": 8192, "len_min": 512, "add": 1, "add_min": 1, "lens": 6},
        # one step of a few very long contexts, in f16, each cut over the whole card
        {"name": "attend_step_long", "op": "attend", "dtype": "f16", "heads": 16, "kv": 2, "dim": 128, "page": 256, "requests": 4,
         "len": 131072, "len_min": 65536, "add": 1, "add_min": 1, "lens": 7},
        # single precision, nothing a power of two, several tokens a request (drafted ones, say), requests with nothing in the cache
        {"name": "attend_odd_f32", "op": "attend", "dtype": "f32", "heads": 6, "kv": 2, "dim": 80, "page": 16, "requests": 9,
         "len": 1333, "len_min": 0, "add": 7, "add_min": 1, "lens": 8},
        # prompts in pieces of 1024 behind what their requests have in the cache already: the largest
        {"name": "attend_prompt", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 8, "dim": 128, "page": 64, "requests": 8,
         "len": 8192, "len_min": 2048, "add": 1024, "add_min": 512, "lens": 9},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["map", "rotary", "store", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    page = rng.choice([16, 32, 64, 128, 256])
    dim = rng.choice([32, 40, 64, 80, 96, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 8, 16])
    lens = rng.randrange(1 << 30)
    if op == "map":
        c = {"op": op, "requests": _log(rng, 1, 1024), "len": _log(rng, 1, 8192), "page": page, "lens": lens}
        c["len_min"] = rng.choice([0, c["len"] // 2])
        c["add"] = rng.choice([1, _log(rng, 1, 1024)])
        c["add_min"] = rng.choice([0, 1])
        return c
    if op == "rotary":
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        return {"op": op, "dtype": dtype, "tokens": _log(rng, 1, 4096), "heads": heads, "kv": kv, "dim": dim, "rot": rot - rot % 2,
                "interleaved": rng.random() < 0.5, "positions": _log(rng, 1024, 1048576), "factor": rng.choice([1.0, 4.0, 32.0]),
                "trained": rng.choice([0, 4096, 8192]), "train": rng.random() < 0.4}
    if op == "store":
        run = rng.choice([1, 100, 1000])                # single tokens, or prompts of up to so many
        return {"op": op, "dtype": dtype, "tokens": _log(rng, 1, 256 if run == 1 else 16384), "kv": kv, "dim": dim, "page": page, "run": run, "lens": lens}
    c = {"op": op, "dtype": dtype, "heads": heads, "kv": kv, "dim": dim, "page": page, "requests": _log(rng, 1, 64),
         "len": _log(rng, 16, 32768), "lens": lens}
    c["len_min"] = rng.choice([0, c["len"] // 8, c["len"] // 2])
    c["add"] = rng.choice([1, 1, 4, _log(rng, 2, 1024)])
    c["add"] = min(c["add"], c["len"])
    c["add_min"] = max(1, c["add"] // 2)
    while work(c)["flops"] > 2e11 or c["requests"] * c["len"] * kv * dim > 6e8 or c["requests"] * c["add"] * heads * c["len"] > 1e9:
        if c["requests"] > 1:                           # no more than the largest listed case, nor than its plain form has room for
            c["requests"] //= 2
        else:
            c["len"], c["len_min"], c["add"] = c["len"] // 2, c["len_min"] // 2, max(1, c["add"] // 2)
            c["add_min"] = max(1, c["add"] // 2)
    return c


def _lengths(case):
    """(tokens in the cache before, tokens added) of every request"""
    r = random.Random(case["lens"])
    have = [r.randint(case["len_min"], case["len"]) for _ in range(case["requests"])]
    add = [r.randint(case["add_min"], case["add"]) for _ in range(case["requests"])]
    return have, add


def _attend_lengths(case):
    """(tokens in the cache, queries) of every request: the queries are the last tokens of the cache; a request whose tokens were dropped
    has queries all the same"""
    length, n = _lengths(case)
    return [0 if x == 0 else max(x, q) for x, q in zip(length, n)], n


def _need(tokens, page):
    return -(-tokens // page)


def work(case):
    op = case["op"]
    if op == "map":
        have, add = _lengths(case)
        new = sum(_need(a + b, case["page"]) - _need(a, case["page"]) for a, b in zip(have, add))
        return {"bytes": 4 * (4 * case["requests"] + 2 * new + 2 * sum(add) + 3), "flops": 2 * sum(add)}
    size = 4 if case["dtype"] == "f32" else 2
    if op == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv"])
        passes = 2 if case["train"] else 1
        return {"bytes": passes * (2 * n * case["dim"] * size + 4 * case["tokens"]), "flops": passes * 3 * n * case["rot"]}
    row = 2 * case["kv"] * (case["dim"] // 2 + -(-case["dim"] // BLOCK))         # a token of the cache
    if op == "store":                                   # in, to the pages, from the pages, out
        return {"bytes": case["tokens"] * (4 * case["kv"] * case["dim"] * size + 2 * row + 8), "flops": 8 * case["tokens"] * case["kv"] * case["dim"]}
    length, n = _attend_lengths(case)
    pairs = sum(sum(max(0, x - q + i + 1) for i in range(q)) for x, q in zip(length, n))
    return {"bytes": sum(length) * row + 2 * sum(n) * case["heads"] * case["dim"] * size + 4 * sum(n) * case["heads"],
            "flops": 4 * case["dim"] * pairs * case["heads"]}


# ---- four bits, in plain form -----------------------------------------------------------------------------------------------

_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]      # halfway; a tie goes to the even code, below at 0.25, 1.25, 2.5, 5, above at the others


def _quantise(x):
    """(.., d) -> codes in 0 .. 15 (.., blocks, 32) uint8, exponents + 127 (.., blocks) uint8; the last block filled up with zeros."""
    d = x.shape[-1]
    x = torch.nn.functional.pad(x.float(), (0, -d % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(EXP_MIN, EXP_MAX)
    y = torch.ldexp(x.abs(), -e[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    for k, b in enumerate(_BORDERS):
        code += (y >= b if k % 2 else y > b).to(torch.uint8)
    return code | (torch.signbit(x).to(torch.uint8) << 3), (e + 127).to(torch.uint8)


def _values(code, scale, d):
    """What codes and scales stand for, in 32 bits: (.., d)."""
    table = torch.tensor(_LEVELS + [-v for v in _LEVELS], device=code.device)
    x = table[code.int()] * torch.exp2(scale.float() - 127)[..., None]
    return x.flatten(-2)[..., :d]


def _nibbles(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _codes(packed):
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2)


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _map_inputs(case, seed):
    have, add = _lengths(case)
    page = case["page"]
    held, need = [_need(x, page) for x in have], [_need(a + b, page) for a, b in zip(have, add)]
    pages = sum(need) + 5
    order = torch.randperm(pages, generator=_generator(seed), device="cuda").int()
    width = max(max(need), 1) + 2
    table = torch.full((case["requests"], width), -1, dtype=torch.int32, device="cuda")
    r = torch.arange(case["requests"], device="cuda").repeat_interleave(torch.tensor(held, device="cuda"))
    first = torch.tensor(held, device="cuda").cumsum(0) - torch.tensor(held, device="cuda")
    table[r, torch.arange(r.numel(), device="cuda") - first[r]] = order[:sum(held)]
    # the list of pages to hand out, of which three have been
    free = torch.cat([order[:3], order[sum(held):]])
    return dict(case=case, lengths=_ints(have), added=_ints(add), free=free, taken=_ints([3]), table=table, pages=pages, tokens=sum(add))


def _turns(case):
    """Frequencies in radians a position, in 64 bits on the host: 10000^(-2 j / rot), those of fewer than one turn in the trained length
    divided by the factor, of more than 32 kept, between mixed by their number of turns; all divided where no length is given."""
    out = []
    for j in range(case["rot"] // 2):
        f = 10000.0 ** (-2.0 * j / case["rot"])
        keep = min(1.0, max(0.0, (case["trained"] * f / (2 * math.pi) - 1.0) / 31.0)) if case["trained"] else 0.0
        out.append((1 - keep) * f / case["factor"] + keep * f)
    return torch.tensor(out, dtype=torch.float64)


def _rotary_inputs(case, seed):
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    position = torch.randint(0, case["positions"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
    names = ("Q", "K") + (("dQ", "dK") if case["train"] else ())
    s = {n: torch.randn(case["tokens"], case["kv"] if n[-1] == "K" else case["heads"], case["dim"], generator=g, device="cuda").to(dt) for n in names}
    return dict(case=case, position=position, scale=1.0 + 0.1 * math.log(case["factor"]), **s)


def _rows(shape, dt, g):
    """Keys or values: normal numbers, some channels larger than others."""
    return (torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-2, 3, shape[1:], generator=g, device="cuda").float())).to(dt)


def _stretches(case):
    """Slots as if the pages were in order, in stretches of a request each that begin anywhere in a page, and the number of pages."""
    r, P = random.Random(case["lens"]), case["page"]
    used, left, out = 0, case["tokens"], []
    while left:
        n, begin = min(left, r.randint(1, case["run"])), used * P + r.randrange(P)
        out.append((begin, n))
        used, left = _need(begin + n, P), left - n
    return out, used + 5


def _store_inputs(case, seed):
    g, dt, P = _generator(seed), DTYPES[case["dtype"]], case["page"]
    shape = (case["tokens"], case["kv"], case["dim"])
    stretches, pages = _stretches(case)
    order = torch.randperm(pages, generator=g, device="cuda")
    begin, n = torch.tensor(stretches, device="cuda").unbind(1)
    at = (begin - n.cumsum(0) + n).repeat_interleave(n) + torch.arange(case["tokens"], device="cuda")
    return dict(case=case, pages=pages, K=_rows(shape, dt, g), V=_rows(shape, dt, g), slots=(order[at // P] * P + at % P).int())


def _attend_inputs(case, seed):
    g, dt, P, G, d = _generator(seed), DTYPES[case["dtype"]], case["page"], case["kv"], case["dim"]
    length, n = _attend_lengths(case)
    need = [_need(x, P) for x in length]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((case["requests"], max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    held = torch.tensor(need, device="cuda")
    r = torch.arange(case["requests"], device="cuda").repeat_interleave(held)
    table[r, torch.arange(r.numel(), device="cuda") - (held.cumsum(0) - held)[r]] = order[:r.numel()]
    start = [0]
    for q in n:
        start.append(start[-1] + q)
    s = dict(case=case, table=table, pages=pages, lengths=_ints(length), start=_ints(start), scale=d ** -0.5,
             Q=torch.randn(start[-1], case["heads"], d, generator=g, device="cuda").to(dt))
    for name in "KV":
        code = torch.empty(pages * P, G, _need(d, BLOCK), BLOCK // 2, dtype=torch.uint8, device="cuda")
        scale = torch.empty(pages * P, G, _need(d, BLOCK), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (G * d))
        larger = torch.exp2(torch.randint(-2, 3, (G, d), generator=g, device="cuda").float()) if name == "K" else 1.0
        for a in range(0, pages * P, step):
            b = min(a + step, pages * P)
            c, e = _quantise(torch.randn(b - a, G, d, generator=g, device="cuda") * larger)
            code[a:b], scale[a:b] = _nibbles(c), e
        s[name] = code, scale
    return s


_INPUTS = {"map": _map_inputs, "rotary": _rotary_inputs, "store": _store_inputs, "attend": _attend_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "rotary":
        s["frequencies"] = _turns(case).cuda()
    if not own:
        if case["op"] == "store":
            blocks = _need(case["dim"], BLOCK)
            s["pages_of"] = {n: [torch.zeros(s["pages"] * case["page"], case["kv"], blocks, *last, dtype=torch.uint8, device="cuda")
                                 for last in ((BLOCK // 2,), ())] for n in "KV"}
        return s
    import paper_2202_04305_amd as sp
    if case["op"] == "rotary":
        s["frequencies"] = sp.sp_rotary_frequencies(case["rot"], 10000.0, factor=case["factor"], trained=case["trained"], low=1.0, high=32.0)
    if case["op"] == "store":
        s["cache"] = sp.sp_cache(s["pages"], case["page"], case["kv"], case["dim"])
    if case["op"] == "attend":
        # the pages as the steps before have left them
        s["cache"] = sp.sp_cache(s["pages"], case["page"], case["kv"], case["dim"])
        slots, step = s["pages"] * case["page"], max(1, (1 << 26) // (case["kv"] * case["dim"]))
        for a in range(0, slots, step):
            b = min(a + step, slots)
            rows = [_values(_codes(s[n][0][a:b]), s[n][1][a:b], case["dim"]).bfloat16() for n in "KV"]
            sp.sp_cache_store(s["cache"], rows[0], rows[1], torch.arange(a, b, dtype=torch.int32, device="cuda"))
        del s["K"], s["V"]
    return s


# ---- the framework's operators ----------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2202_04305_amd as sp
    case = s["case"]
    if case["op"] == "map":
        lengths, start, position, slot, taken = sp.sp_cache_map(s["lengths"], s["added"], s["free"], s["taken"], s["table"], case["page"], s["pages"], s["tokens"])
        return {"lengths": lengths, "start": start, "position": position, "slot": slot, "taken": taken, "table": s["table"]}
    if case["op"] == "rotary":
        more = {"interleaved": case["interleaved"], "scale": s["scale"]}
        Q, K = sp.sp_rotary(s["position"], s["frequencies"], s["Q"], s["K"], **more)
        if not case["train"]:
            return {"Q": Q, "K": K}
        dQ, dK = sp.sp_rotary_grad(s["position"], s["frequencies"], s["dQ"], s["dK"], **more)
        return {"Q": Q, "K": K, "dQ": dQ, "dK": dK}
    if case["op"] == "store":
        sp.sp_cache_store(s["cache"], s["K"], s["V"], s["slots"])
        K, V = sp.sp_cache_load(s["cache"], s["slots"], s["K"].dtype)
        return {"K": K, "V": V}
    O, lse = sp.sp_cache_attention(s["cache"], s["Q"], s["table"], s["lengths"], s["start"], scale=s["scale"], causal=True)
    return {"O": O, "lse": lse}


# ---- the plain forms --------------------------------------------------------------------------------------------------------

def _map_plain(s):
    case, P = s["case"], s["case"]["page"]
    have, add, table, free = s["lengths"].long(), s["added"].long(), s["table"], s["free"]
    held = (have + P - 1) // P
    new = (have + add + P - 1) // P - held
    ends, page_ends = add.cumsum(0), new.cumsum(0)
    # pages: a request's place in the list, then its place in the request
    k = torch.arange(table.shape[1], device=table.device)
    j = k[None, :] - held[:, None]
    at = (s["taken"].long() + page_ends - new)[:, None] + j
    table.copy_(torch.where((j >= 0) & (j < new[:, None]), free[at.clamp(0, free.numel() - 1)], table))
    i = torch.arange(s["tokens"], device=table.device)
    r = torch.searchsorted(ends, i, right=True)
    position = have[r] + i - (ends - add)[r]
    slot = table[r, position // P].long() * P + position % P
    start = torch.cat([torch.zeros_like(ends[:1]), ends])
    return {"lengths": (have + add).int(), "start": start.int(), "position": position.int(), "slot": slot.int(),
            "taken": (s["taken"].long() + page_ends[-1]).int(), "table": table}


def _rotate(x, angle, case, scale, back):
    rot = case["rot"]
    c, n = (torch.cos(angle) * scale).float()[:, None], (torch.sin(angle) * (-scale if back else scale)).float()[:, None]
    y = x.float().clone()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    p, q = a * c - b * n, a * n + b * c
    if case["interleaved"]:
        y[..., 0:rot:2], y[..., 1:rot:2] = p, q
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = p, q
    return y.to(x.dtype)


def _rotary_plain(s):
    case = s["case"]
    angle = s["position"].double()[:, None] * s["frequencies"]
    out = {n: _rotate(s[n], angle, case, s["scale"], False) for n in ("Q", "K")}
    if case["train"]:
        out.update({n: _rotate(s[n], angle, case, s["scale"], True) for n in ("dQ", "dK")})
    return out


def _store_plain(s):
    at = s["slots"].long()
    for n in "KV":
        code, scale = _quantise(s[n])
        s["pages_of"][n][0][at], s["pages_of"][n][1][at] = _nibbles(code), scale
    return {n: _values(_codes(s["pages_of"][n][0][at]), s["pages_of"][n][1][at], s["case"]["dim"]).to(s[n].dtype) for n in "KV"}


def _attend_plain(s):
    case, P, H, G, d = s["case"], s["case"]["page"], s["case"]["heads"], s["case"]["kv"], s["case"]["dim"]
    length, start, table = s["lengths"].long(), s["start"].long(), s["table"].long()
    n = start[1:] - start[:-1]
    R, r, Lmax, Lq = case["requests"], H // G, table.shape[1] * P, case["add"]
    t, i = torch.arange(Lmax, device=table.device), torch.arange(Lq, device=table.device)
    slot = table.clamp(min=0)[:, t // P] * P + t % P
    rows = (start[:-1, None] + i).clamp(max=s["Q"].shape[0] - 1)
    there = i < n[:, None]

    def gathered(name):                                 # (R, kv, Lmax, d)
        return _values(_codes(s[name][0][slot]), s[name][1][slot], d).transpose(1, 2).contiguous()
    q = s["Q"].float()[rows].view(R, Lq, G, r, d).permute(0, 2, 3, 1, 4).reshape(R, G, r * Lq, d)
    sc = torch.matmul(q, gathered("K").transpose(-1, -2)).view(R, G, r, Lq, Lmax) * s["scale"]
    keep = (t[None, None, :] <= (length - n)[:, None, None] + i[None, :, None]) & (t < length[:, None])[:, None, :]
    sc = sc.masked_fill(~keep[:, None, None], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    e = torch.exp(sc - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    p = e / torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(R, G, r * Lq, Lmax), gathered("V")).view(R, G, r, Lq, d)
    return {"O": o.permute(0, 3, 1, 2, 4)[there].reshape(-1, H, d).to(s["Q"].dtype),
            "lse": lse[..., 0].permute(0, 3, 1, 2)[there].reshape(-1, H).t().contiguous()}


_PLAIN = {"map": _map_plain, "rotary": _rotary_plain, "store": _store_plain, "attend": _attend_plain}


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- the definitions, in 64 bits --------------------------------------------------------------------------------------------

def _map_exact(s):
    case, P = s["case"], s["case"]["page"]
    have, add, free = s["lengths"].tolist(), s["added"].tolist(), s["free"].tolist()
    taken, table = s["taken"].item(), s["table"].cpu().numpy().copy()
    start, position, slot, after = [0], [], [], []
    for r, (a, b) in enumerate(zip(have, add)):
        for t in range(a, a + b):
            if t % P == 0:
                table[r, t // P] = free[taken]
                taken += 1
            position.append(t)
            slot.append(int(table[r, t // P]) * P + t % P)
        start.append(start[-1] + b)
        after.append(a + b)
    return {"lengths": _ints(after), "start": _ints(start), "position": _ints(position), "slot": _ints(slot), "taken": _ints([taken]),
            "table": torch.from_numpy(table).cuda()}


def _rotary_exact(s):
    case, half = s["case"], s["case"]["rot"] // 2
    out = {}
    z = torch.polar(torch.full((1, 1), s["scale"], dtype=torch.float64, device="cuda"), s["position"].double()[:, None] * _turns(case).cuda())[:, None]
    for n in ("Q", "K") + (("dQ", "dK") if case["train"] else ()):
        x = s[n].double()
        pairs = x[..., :2 * half].unflatten(-1, (half, 2)) if case["interleaved"] else x[..., :2 * half].unflatten(-1, (2, half)).transpose(-1, -2)
        w = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * (z.conj() if n[0] == "d" else z))
        w = w if case["interleaved"] else w.transpose(-1, -2)
        out[n] = torch.cat([w.flatten(-2), x[..., 2 * half:]], -1)
    return out


def _store_exact(s):
    def nearest(x):
        d = x.shape[-1]
        out = torch.empty_like(x)
        levels = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
        even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)
        for a in range(0, d, BLOCK):
            b = x[..., a:a + BLOCK]
            top = b.abs().amax(-1, keepdim=True)
            e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 7)), torch.full_like(top, -200.0))
            e = torch.where(top > 7 * torch.exp2(e), e + 1, e)
            e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e).clamp(EXP_MIN, EXP_MAX)
            y = b.abs() / torch.exp2(e)
            best = torch.full_like(y, math.inf)
            value = torch.zeros_like(y)
            for k in even_first.tolist():               # of two that are as near, the even one comes first
                off = (y - levels[k]).abs()
                value = torch.where(off < best, levels[k], value)
                best = torch.minimum(off, best)
            out[..., a:a + BLOCK] = torch.copysign(value * torch.exp2(e), b)
        return out
    return {n: nearest(s[n].double()) for n in ("K", "V")}


def _attend_exact(s):
    case, P, H, G, d = s["case"], s["case"]["page"], s["case"]["heads"], s["case"]["kv"], s["case"]["dim"]
    O, lse = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda"), torch.full((H, s["Q"].shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    start = s["start"].tolist()

    def stored(name, slot, g):                          # sign, two bits of exponent, one of fraction
        byte = s[name][0][slot, g].long()
        code = torch.stack([byte % 16, byte // 16], -1).reshape(slot.numel(), -1, BLOCK)
        e, f = (code % 8) // 2, (code % 2).double()
        v = torch.where(e == 0, f / 2, (1 + f / 2) * torch.exp2((e - 1).double()))
        v = torch.where(code >= 8, -v, v) * torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), s[name][1][slot, g].double() - 127)[..., None]
        return v.reshape(slot.numel(), -1)[:, :d].contiguous()
    for z, L in enumerate(s["lengths"].tolist()):
        a, b = start[z], start[z + 1]
        if L == 0 or a == b:
            continue
        slot = (s["table"][z, :_need(L, P)].long()[:, None] * P + torch.arange(P, device="cuda")).reshape(-1)[:L]
        late = torch.arange(L, device="cuda")[None, :] > torch.arange(L - (b - a), L, device="cuda")[:, None]
        for g in range(G):
            K, V = stored("K", slot, g), stored("V", slot, g)
            Kt = K.t().contiguous()
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = (torch.mm(s["Q"][a:b, h].double(), Kt) * s["scale"]).masked_fill(late, -math.inf)
                w = torch.logsumexp(x, 1)
                lse[h, a:b] = w
                O[a:b, h] = torch.mm(torch.exp(x - torch.where(torch.isinf(w), torch.zeros_like(w), w)[:, None]), V)
    return {"O": O, "lse": lse}


_EXACT = {"map": _map_exact, "rotary": _rotary_exact, "store": _store_exact, "attend": _attend_exact}


def exact(case, seed):
    return _EXACT[case["op"]](_INPUTS[case["op"]](case, seed))
