"""Attention over a stored pattern, as measurable cases: queries are the rows and keys the columns of a sparse matrix, and a query
attends to the columns its row stores.  Cross attention of a ragged batch to encoder states of another length, a batch of single
tokens that shares a long prefix, attention with a learned relative position bias by buckets, and their gradients.

A case is a dict of plain values.  `kind` says the direction (`forward`, or `train`: forward and gradients); `pattern` how the
stored positions lie; `lens` seeds the lengths of the sequences, so that the work of a case does not depend on the seed of its
inputs.

The plain form knows the pattern as groups of rows that attend to a list of columns each (with a mask), and columns that every row
attends to: two batched products with a softmax between them, in 32 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BAND = 128          # rows of a group of the band pattern


def listed():
    return [
        # one decoding step of a small batch that attends to short encoder states: launches and host work are all there is
        {"name": "cross_step_small", "kind": "forward", "pattern": "batch", "dtype": "bf16", "heads": 8, "kv": 8, "dim": 64, "batch": 4,
         "lq": 1, "lq_min": 1, "lk": 200, "lk_min": 64, "lens": 1},
        # one decoding step of a serving batch over the encoder states of audio or documents
        {"name": "cross_step_batch", "kind": "forward", "pattern": "batch", "dtype": "f16", "heads": 16, "kv": 16, "dim": 64, "batch": 64,
         "lq": 1, "lq_min": 1, "lk": 1500, "lk_min": 800, "lens": 2},
        # whole target sequences against long encoder states, grouped heads: the largest forward pass
        {"name": "cross_prefill", "kind": "forward", "pattern": "batch", "dtype": "bf16", "heads": 16, "kv": 4, "dim": 128, "batch": 16,
         "lq": 1024, "lq_min": 512, "lk": 4096, "lk_min": 2048, "lens": 3},
        # single precision, nothing a power of two, sequences without any encoder state
        {"name": "cross_odd_f32", "kind": "forward", "pattern": "batch", "dtype": "f32", "heads": 6, "kv": 2, "dim": 80, "batch": 9,
         "lq": 211, "lq_min": 37, "lk": 333, "lk_min": 0, "lens": 4},
        # every query attends to a few retrieved states among many: no two queries share much
        {"name": "cross_scattered", "kind": "forward", "pattern": "scattered", "dtype": "bf16", "heads": 8, "kv": 8, "dim": 64, "rows": 4096,
         "cols": 65536, "per_row": 96, "lens": 5},
        # a training step of a decoder's cross attention
        {"name": "cross_train", "kind": "train", "pattern": "batch", "dtype": "bf16", "heads": 12, "kv": 12, "dim": 64, "batch": 16,
         "lq": 512, "lq_min": 256, "lk": 1024, "lk_min": 512, "lens": 6},
        # the same in single precision at small odd sizes (fine-tuning, checks of gradients)
        {"name": "cross_train_f32", "kind": "train", "pattern": "batch", "dtype": "f32", "heads": 4, "kv": 2, "dim": 40, "batch": 5,
         "lq": 203, "lq_min": 101, "lk": 307, "lk_min": 0, "lens": 7},
        # a training step of an encoder with a learned position bias (both directions, 32 buckets up to a distance of 128)
        {"name": "bias_train", "kind": "train", "pattern": "self", "dtype": "bf16", "heads": 12, "kv": 12, "dim": 64, "batch": 16,
         "lq": 512, "lq_min": 200, "lens": 8, "buckets": 32, "max_distance": 128, "bidirectional": True},
        # a training step over one long document: a band of 256 to each side and 32 columns that all rows attend to
        {"name": "bias_band_train", "kind": "train", "pattern": "band", "dtype": "bf16", "heads": 12, "kv": 12, "dim": 64, "rows": 16384,
         "width": 256, "shared": 32, "lens": 9, "buckets": 32, "max_distance": 128, "bidirectional": True},
        # one decoding step with the bias: caches with room for 1024 tokens, of which the positions say how many count
        {"name": "bias_step", "kind": "forward", "pattern": "cache", "dtype": "f16", "heads": 16, "kv": 16, "dim": 64, "batch": 32,
         "lk": 1024, "lk_min": 100, "lens": 10, "buckets": 32, "max_distance": 128, "bidirectional": False},
        # a few samples of one prompt
        {"name": "prefix_small", "kind": "forward", "pattern": "prefix", "dtype": "bf16", "heads": 16, "kv": 2, "dim": 128, "batch": 8,
         "shared": 1000, "lk": 60, "lk_min": 1, "lens": 11},
        # many requests behind one long system prompt: the largest single-token step
        {"name": "prefix_long", "kind": "forward", "pattern": "prefix", "dtype": "bf16", "heads": 32, "kv": 8, "dim": 128, "batch": 64,
         "shared": 32768, "lk": 1024, "lk_min": 64, "lens": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kv = rng.choice([1, 2, 4, 8])
    c = {"kind": "forward", "pattern": rng.choice(["batch", "batch", "scattered", "self", "band", "cache", "prefix"]),
         "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "heads": kv * rng.choice([1, 1, 2, 3, 4, 8]), "kv": kv,
         "dim": rng.choice([32, 40, 64, 64, 80, 128, 128]), "lens": rng.randrange(1 << 30)}
    p = c["pattern"]
    if p in ("batch", "self"):
        c["kind"] = rng.choice(["forward", "train"])
        step = p == "batch" and c["kind"] == "forward" and rng.random() < 0.4
        c["batch"] = _log(rng, 1, 64 if step else 16)
        c["lq"] = 1 if step else _log(rng, 16, 1024)
        c["lq_min"] = max(1, c["lq"] // 2)
        if p == "batch":
            c["lk"] = _log(rng, 33, 4096 if step or c["kind"] == "forward" else 2048)
            c["lk_min"] = rng.choice([0, c["lk"] // 2, c["lk"]])
    elif p == "scattered":
        c["rows"], c["cols"] = _log(rng, 64, 4096), _log(rng, 4096, 65536)
        c["per_row"] = _log(rng, 8, 128)
    elif p == "band":
        c["kind"] = rng.choice(["forward", "train"])
        c["rows"], c["width"], c["shared"] = _log(rng, 1000, 16384), _log(rng, 16, 256), rng.choice([0, 1, 32])
    elif p == "cache":
        c["batch"], c["lk"] = _log(rng, 1, 64), _log(rng, 64, 2048)
        c["lk_min"] = max(1, c["lk"] // 8)
    else:
        c["batch"], c["shared"], c["lk"] = _log(rng, 2, 64), _log(rng, 500, 32768), _log(rng, 2, 1024)
        c["lk_min"] = 1
    if p in ("self", "band", "cache"):
        c["buckets"], c["max_distance"] = rng.choice([16, 32, 64]), rng.choice([64, 128, 200])
        c["bidirectional"] = p != "cache"
    while work(c)["flops"] > 3e11:                      # no more than the largest listed case
        less = "batch" if "batch" in c else "rows"
        c[less] = max(1, c[less] // 2)
    return c


def _lengths(case):
    """(queries, keys) of every sequence."""
    r = random.Random(case["lens"])
    if case["pattern"] in ("batch", "self"):
        lq = [r.randint(case["lq_min"], case["lq"]) for _ in range(case["batch"])]
        lk = lq if case["pattern"] == "self" else [r.randint(case["lk_min"], case["lk"]) for _ in range(case["batch"])]
    else:                                               # single tokens
        lq, lk = [1] * case["batch"], [r.randint(case["lk_min"], case["lk"]) for _ in range(case["batch"])]
    return lq, lk


def _sizes(case):
    """(queries, keys, attended pairs)"""
    p = case["pattern"]
    if p == "scattered":
        return case["rows"], case["cols"], case["rows"] * case["per_row"]
    if p == "band":
        m, w, g = case["rows"], case["width"], case["shared"]
        pairs = sum(min(m, i + w + 1) - max(0, i - w) + max(0, min(g, i - w)) for i in range(m))
        return m, m, pairs
    lq, lk = _lengths(case)
    if p == "cache":
        return sum(lq), case["batch"] * case["lk"], sum(lk)
    if p == "prefix":
        return sum(lq), case["shared"] + sum(lk), case["batch"] * case["shared"] + sum(lk)
    return sum(lq), sum(lk), sum(a * b for a, b in zip(lq, lk))


def work(case):
    m, n, pairs = _sizes(case)
    size = 4 if case["dtype"] == "f32" else 2
    rows, cols = m * case["heads"] * case["dim"] * size, n * case["kv"] * case["dim"] * size
    table = case.get("buckets", 0) * case["heads"] * size
    if case["pattern"] == "cache":                      # of the caches, only what the positions leave
        cols = pairs * case["kv"] * case["dim"] * size
    bytes_ = 2 * rows + 2 * cols + 4 * m * case["heads"] + table
    flops = 4 * case["dim"] * pairs * case["heads"]
    if case["kind"] == "train":                         # dO in; dQ, dK, dV and the table's gradient out; five more products
        bytes_ += 2 * rows + 2 * cols + table
        flops += 10 * case["dim"] * pairs * case["heads"]
    return {"bytes": bytes_, "flops": flops}


def _layout(case, g, dev):
    """The pattern: rows (G, Lq) and cols (G, Lk) of every group with their masks, cols_all of every row, positions."""
    p = case["pattern"]
    if p == "scattered":
        m, n, k = case["rows"], case["cols"], case["per_row"]
        # one column of each of k stretches of the row's own cut: distinct and ascending
        cut = (torch.arange(k, device=dev) * n) // k
        wide = (torch.arange(1, k + 1, device=dev) * n) // k - cut
        cols = cut + (torch.rand(m, k, generator=g, device=dev, dtype=torch.float64) * wide).long()
        rows = torch.arange(m, device=dev).view(m, 1)
        mask = torch.ones(m, 1, k, dtype=torch.bool, device=dev)
        return dict(m=m, n=n, rows=rows, cols=cols, mask=mask, rmask=torch.ones_like(rows, dtype=torch.bool), shared=0, qpos=None, kpos=None)
    if p == "band":
        m, w, s = case["rows"], case["width"], case["shared"]
        G = -(-m // BAND)
        rows = torch.arange(G * BAND, device=dev).view(G, BAND)
        cols = torch.arange(G, device=dev).view(G, 1) * BAND - w + torch.arange(BAND + 2 * w, device=dev)
        mask = (rows[:, :, None] - cols[:, None, :]).abs() <= w
        mask &= ((cols >= s) & (cols < m))[:, None, :] & (rows < m)[:, :, None]
        pos = torch.arange(m, device=dev, dtype=torch.int32)
        return dict(m=m, n=m, rows=rows.clamp(max=m - 1), cols=cols.clamp(0, m - 1), mask=mask, rmask=rows < m, shared=s, qpos=pos, kpos=pos)
    lq, lk = (torch.tensor(v, device=dev) for v in _lengths(case))
    s = case["shared"] if p == "prefix" else 0
    room = torch.full_like(lk, case["lk"]) if p == "cache" else lk
    iq, ik = torch.arange(int(lq.max()), device=dev), torch.arange(max(1, int(room.max())), device=dev)
    rmask, cmask = iq < lq[:, None], ik < room[:, None]
    rows, cols = (lq.cumsum(0) - lq)[:, None] + iq, s + (room.cumsum(0) - room)[:, None] + ik
    m, n = int(lq.sum()), s + int(room.sum())
    mask = rmask[:, :, None] & cmask[:, None, :]
    qpos = kpos = None
    if p == "self":
        qpos = kpos = iq.expand(rmask.shape)[rmask].to(torch.int32)
    if p == "cache":                                    # the token at position lk - 1 has just been appended
        qpos, kpos = (lk - 1).to(torch.int32), ik.expand(cmask.shape)[cmask].to(torch.int32)
    return dict(m=m, n=n, rows=rows.clamp(max=m - 1), cols=cols.clamp(max=max(0, n - 1)), mask=mask, rmask=rmask, shared=s, qpos=qpos, kpos=kpos)


def _inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    s = _layout(case, g, dev)
    dt, d = DTYPES[case["dtype"]], case["dim"]

    def normal(rows, heads):
        return torch.randn(rows, heads, d, generator=g, device=dev).to(dt)
    s["Q"], s["K"], s["V"] = normal(s["m"], case["heads"]), normal(s["n"], case["kv"]), normal(s["n"], case["kv"])
    s["dO"] = normal(s["m"], case["heads"]) if case["kind"] == "train" else None
    s["table"] = torch.randn(case["buckets"], case["heads"], generator=g, device=dev).to(dt) if "buckets" in case else None
    s["case"], s["scale"], s["causal"] = case, d ** -0.5, case["pattern"] == "cache"
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # the packed pattern, looked at once: a program keeps it for all layers and steps of these sequences
        import paper_2202_04305_amd as sp
        m, n = s["m"], s["n"]
        at = s["mask"].nonzero(as_tuple=True)
        rows, cols = s["rows"][at[0], at[1]], s["cols"][at[0], at[2]]
        if s["shared"]:
            rows = torch.cat([rows, torch.arange(m, device=rows.device).repeat_interleave(s["shared"])])
            cols = torch.cat([cols, torch.arange(s["shared"], device=rows.device).repeat(m)])
        ones = torch.ones(rows.numel(), dtype=torch.float32, device=rows.device)
        s["S"] = sp.sp_pack(sp.sp_encode((sp.SP_DENSE, sp.SP_COMPRESSED), None, 32, 32), (m, n), [rows.contiguous(), cols.contiguous()], ones)
        sp.sp_prepare_attention(s["S"], grad=case["kind"] == "train")
    return s


def _run_own(s):
    import paper_2202_04305_amd as sp
    case, more = s["case"], {"scale": s["scale"]}
    if s["table"] is not None:
        more.update(qpos=s["qpos"], kpos=s["kpos"], bias=s["table"], max_distance=case["max_distance"],
                    bidirectional=case["bidirectional"], causal=s["causal"])
    O, lse = sp.sp_attention(s["S"], s["Q"], s["K"], s["V"], **more)
    if case["kind"] != "train":
        return {"O": O, "lse": lse}
    dQ, dK, dV, dT = sp.sp_attention_grad(s["S"], s["Q"], s["K"], s["V"], O, lse, s["dO"], **more)
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV, **({} if dT is None else {"dT": dT})}


def _bucket(rel, case):
    """The bucket of a key at distance rel = key's position - query's."""
    side, base = case["buckets"], 0
    if case["bidirectional"]:
        side //= 2
        base = (rel > 0) * side
        d = rel.abs()
    else:
        d = (-rel).clamp(min=0)
    exact = side // 2
    far = torch.log(d.clamp(min=1).double() / exact) * ((side - exact) / math.log(case["max_distance"] / exact))
    far = (exact + torch.floor(far + 1e-9).long()).clamp(max=side - 1)
    return base + torch.where(d < exact, d.long(), far)


def _run_plain(s):
    case, f = s["case"], torch.float32
    H, Hk, D = case["heads"], case["kv"], case["dim"]
    r, shared = H // Hk, s["shared"]
    rows, cols, mask = s["rows"], s["cols"], s["mask"]
    G, Lq, Lk = mask.shape
    # (G, kv, r * Lq, D) queries; (G, kv, Lk, D) keys and values of the groups; (kv, shared, D) of all

    def split(x):
        return x.to(f)[rows].view(G, Lq, Hk, r, D).permute(0, 2, 3, 1, 4).reshape(G, Hk, r * Lq, D)

    def own_cols(x):
        return x.to(f)[cols].permute(0, 2, 1, 3).contiguous()

    def all_cols(x):
        return x[:shared].to(f).transpose(0, 1).contiguous()

    def to_all(x):                                      # (G, kv, r * Lq, D) -> (kv, G * r * Lq, D)
        return x.transpose(0, 1).reshape(Hk, G * r * Lq, -1)

    def from_all(x):
        return x.view(Hk, G, r * Lq, -1).transpose(0, 1)

    q, k, v = split(s["Q"]), own_cols(s["K"]), own_cols(s["V"])
    sc = torch.matmul(q, k.transpose(-1, -2))
    keep = mask
    if shared:
        ka, va = all_cols(s["K"]), all_cols(s["V"])
        sc = torch.cat([from_all(torch.matmul(to_all(q), ka.transpose(-1, -2))), sc], -1)
        keep = torch.cat([s["rmask"][:, :, None].expand(G, Lq, shared), mask], -1)
    sc = sc.view(G, Hk, r, Lq, shared + Lk) * s["scale"]
    if s["table"] is not None:
        places = torch.cat([torch.arange(shared, device=cols.device).expand(G, shared), cols], -1)
        rel = s["kpos"][places].long()[:, None, :] - s["qpos"][rows].long()[:, :, None]
        bucket = _bucket(rel, case)
        sc = sc + s["table"].to(f)[bucket].permute(0, 3, 1, 2).view(G, Hk, r, Lq, shared + Lk)
        if s["causal"]:
            keep = keep & (rel <= 0)
    sc = sc.masked_fill(~keep[:, None, None], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    e = torch.exp(sc - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).view(G, H, Lq)
    p = (e / torch.where(total == 0, torch.ones_like(total), total)).view(G, Hk, r * Lq, shared + Lk)
    o = torch.matmul(p[..., shared:], v)
    if shared:
        o = o + from_all(torch.matmul(to_all(p[..., :shared].contiguous()), va))
    there = s["rmask"]

    def join(x):                                        # (G, kv, r * Lq, D) -> (m, H, D)
        return x.view(G, Hk, r, Lq, D).permute(0, 3, 1, 2, 4)[there].reshape(s["m"], H, D)

    out = {"O": join(o).to(s["Q"].dtype), "lse": lse.permute(0, 2, 1)[there].t().contiguous()}
    if case["kind"] != "train":
        return out
    do = split(s["dO"])
    dp = torch.matmul(do, v.transpose(-1, -2))
    if shared:
        dp = torch.cat([from_all(torch.matmul(to_all(do), va.transpose(-1, -2))), dp], -1)
    ds = p * (dp - (do * o).sum(-1, keepdim=True))
    pt, dst = p.transpose(-1, -2), ds.transpose(-1, -2)
    dq = torch.matmul(ds[..., shared:], k)
    if shared:
        dq = dq + from_all(torch.matmul(to_all(ds[..., :shared].contiguous()), ka))
    out["dQ"] = join(dq * s["scale"]).to(s["Q"].dtype)
    flat = cols.reshape(-1)

    def sum_cols(at, x, scale):
        d = torch.matmul(at[..., shared:, :], x)                                   # (G, kv, Lk, D)
        total = torch.zeros(s["n"], Hk, D, dtype=f, device=x.device).index_add_(0, flat, d.permute(0, 2, 1, 3).reshape(-1, Hk, D))
        if shared:
            total[:shared] += torch.matmul(to_all(at[..., :shared, :].transpose(-1, -2)).transpose(-1, -2), to_all(x)).transpose(0, 1)
        return (total * scale).to(s["Q"].dtype)
    padded = there[:, None, None, :, None].expand(G, Hk, r, Lq, 1).reshape(G, Hk, r * Lq, 1)
    out["dK"], out["dV"] = sum_cols(dst, q * padded, s["scale"]), sum_cols(pt, do * padded, 1.0)
    if s["table"] is not None:
        # a small product with the buckets as unit vectors for every row, then the rows' sums in 64 bits
        L = shared + Lk
        ones = torch.zeros(G * Lq, L, case["buckets"], dtype=f, device=bucket.device).scatter_(2, bucket.view(G * Lq, L, 1), 1.0)
        each = torch.matmul(ds.view(G, H, Lq, L).transpose(1, 2).reshape(G * Lq, H, L), ones)
        out["dT"] = each.sum(0, dtype=torch.float64).t().to(s["Q"].dtype).contiguous()
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _bucket_by_search(rel, case):
    """The same buckets from their borders: the k-th far bucket begins at the smallest distance d with (d/e)^(N-e) >= (M/e)^k."""
    side = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    e, M = side // 2, case["max_distance"]
    far = side - e
    borders = [next(d for d in range(e, M + 2) if d ** far * e ** k >= M ** k * e ** far) for k in range(1, far)]
    d = rel.abs() if case["bidirectional"] else (-rel).clamp(min=0)
    b = torch.where(d < e, d, e + torch.searchsorted(torch.tensor(borders, device=rel.device), d, right=True))
    return b + (side * (rel > 0) if case["bidirectional"] else 0)


def exact(case, seed):
    """Row by row of the definition in 64 bits: a sequence (a stretch of rows) and a head at a time."""
    if _sizes(case)[2] * case["heads"] * case["dim"] * (14 if case["kind"] == "train" else 4) > 3e12:
        return None
    s = _inputs(case, seed)
    H, r = case["heads"], case["heads"] // case["kv"]
    Q, K, V = (s[x].double().transpose(0, 1).contiguous() for x in "QKV")
    O, lse = torch.zeros_like(Q), torch.full(Q.shape[:2], float("-inf"), dtype=torch.float64, device=Q.device)
    train = case["kind"] == "train"
    if train:
        dO = s["dO"].double().transpose(0, 1).contiguous()
        dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    if s["table"] is not None:
        T, qpos, kpos = s["table"].double(), s["qpos"].long(), s["kpos"].long()
        dT = torch.zeros_like(T)
    G = s["rows"].shape[0]
    # groups of single rows are taken many at a time, as rows over all columns that any of them has
    for a in range(0, G, 1 if s["rows"].shape[1] > 1 else 64):
        z = slice(a, a + (1 if s["rows"].shape[1] > 1 else 64))
        i = s["rows"][z][s["rmask"][z]]
        if i.numel() == 0:
            continue
        j = torch.unique(torch.cat([torch.arange(s["shared"], device=i.device), s["cols"][z].reshape(-1)]))
        if j.numel() == 0 or s["n"] == 0:
            continue
        at = torch.zeros(i.numel(), j.numel(), dtype=torch.bool, device=i.device)
        local = torch.cumsum(s["rmask"][z].reshape(-1).long(), 0).view(s["rmask"][z].shape) - 1
        gi, qi, ci = s["mask"][z].nonzero(as_tuple=True)
        at[local[gi, qi], torch.searchsorted(j, s["cols"][z][gi, ci])] = True
        at[:, j < s["shared"]] = True
        if s["table"] is not None:
            rel = kpos[j][None, :] - qpos[i][:, None]
            b = _bucket_by_search(rel, case)
            if s["causal"]:
                at &= rel <= 0
        for h in range(H):
            g = h // r
            x = torch.mm(Q[h, i], K[g, j].t().contiguous()) * s["scale"]
            if s["table"] is not None:
                x = x + T[:, h][b]
            x = x.masked_fill(~at, float("-inf"))
            L = torch.logsumexp(x, 1)
            p = torch.where(at, torch.exp(x - torch.where(torch.isinf(L), torch.zeros_like(L), L)[:, None]), torch.zeros_like(x))
            lse[h, i], O[h, i] = L, torch.mm(p, V[g, j])
            if train:
                ds = p * (torch.mm(dO[h, i], V[g, j].t().contiguous()) - (dO[h, i] * O[h, i]).sum(1, keepdim=True))
                dQ[h, i] = torch.mm(ds, K[g, j]) * s["scale"]
                dK[g].index_add_(0, j, torch.mm(ds.t().contiguous(), Q[h, i]) * s["scale"])
                dV[g].index_add_(0, j, torch.mm(p.t().contiguous(), dO[h, i]))
                if s["table"] is not None:
                    dT[:, h] += torch.bincount(b.reshape(-1), ds.reshape(-1), minlength=case["buckets"])
    out = {"O": O.transpose(0, 1).contiguous(), "lse": lse}
    if train:
        out.update(dQ=dQ.transpose(0, 1).contiguous(), dK=dK.transpose(0, 1).contiguous(), dV=dV.transpose(0, 1).contiguous())
        if s["table"] is not None:
            out["dT"] = dT
    return out
