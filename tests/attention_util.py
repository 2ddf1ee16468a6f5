"""Attention over a stored pattern in 64 bits on the CPU, from the definition, with the error that the GPU's arithmetic may have.

The bounds count roundings.  u = half a step of the operands' type, v = 2^-24 (f32, in which everything is summed):
  a score s:            (D + 8) v * scale * sum |q||k|, plus 4 v |s| for its scaling, the bias and the base of the power
  a weight p:           twice the largest score error among the row's pairs above e^-200 (its own and the sum's), the sum's (pairs + 8) v, |lse| v
  p as an operand:      u more (16-bit types)
  dp, D:                (D + 8) v of the sums of absolute products; D takes O as it was rounded: u of sum |dO||O|
  ds as an operand:     u
  a result:             u of itself, and (pairs + 8) v of the sum of the absolute terms
"""
import torch


class Problem:
    """Everything one attention call takes, on the CPU.  at: bool (m, n), the stored pairs."""

    def __init__(self, at, Q, K, V, scale=None, causal=False, qpos=None, kpos=None, bias=None, max_distance=128, bidirectional=True, dO=None):
        self.at, self.Q, self.K, self.V, self.dO = at, Q, K, V, dO
        self.scale = Q.shape[2] ** -0.5 if scale is None else scale
        self.causal, self.qpos, self.kpos, self.bias = causal, qpos, kpos, bias
        self.max_distance, self.bidirectional = max_distance, bidirectional

    def options(self, device):
        o = {"scale": self.scale}
        if self.bias is not None or self.causal:
            o.update(qpos=self.qpos.to(device), kpos=self.kpos.to(device), causal=self.causal)
        if self.bias is not None:
            o.update(bias=self.bias.to(device), max_distance=self.max_distance, bidirectional=self.bidirectional)
        return o


def buckets_of(rel, buckets, max_distance, bidirectional):
    """Bucket of every distance, from borders found by whole-number comparison: d >= e (M/e)^(k/(N-e))."""
    side = buckets // 2 if bidirectional else buckets
    e = side // 2
    far = side - e
    borders, d = [], e
    for k in range(1, far):
        while d ** far * e ** k < max_distance ** k * e ** far:
            d += 1
        borders.append(d)
    dist = rel.abs() if bidirectional else (-rel).clamp(min=0)
    b = dist.clone()
    b[dist >= e] = e
    for x in borders:
        b += (dist >= x).long()
    return b + (side * (rel > 0).long() if bidirectional else 0)


def reference(p, grads=True):
    """{name: (value, bound on the GPU's error)} in f64."""
    f = torch.float64
    Q, K, V = (t.to(f) for t in (p.Q, p.K, p.V))
    m, H, D = Q.shape
    n, Hk, _ = K.shape
    r = H // Hk
    dt = p.Q.dtype
    u = torch.finfo(dt).eps / 2
    w16 = u if dt != torch.float32 else 0.0              # f32 operands of a product are not rounded
    v = 2.0 ** -24
    tiny = float(torch.finfo(dt).smallest_normal) if dt != torch.float16 else 2.0 ** -24     # below: rounded away or a step of the subnormals
    at = p.at.clone()
    rel = None
    if p.causal or p.bias is not None:
        rel = p.kpos.long()[None, :] - p.qpos.long()[:, None]
        if p.causal:
            at &= rel <= 0
    out = {"O": torch.zeros(m, H, D, dtype=f), "lse": torch.full((H, m), float("-inf"), dtype=f)}
    tol = {k: torch.zeros_like(t) for k, t in out.items()}
    if grads:
        dO = p.dO.to(f)
        for k, t in (("dQ", Q), ("dK", K), ("dV", V)):
            out[k], tol[k] = torch.zeros_like(t), torch.zeros_like(t)
        if p.bias is not None:
            out["dT"], tol["dT"] = torch.zeros(p.bias.shape, dtype=f), torch.zeros(p.bias.shape, dtype=f)
    bucket = buckets_of(rel, p.bias.shape[0], p.max_distance, p.bidirectional) if p.bias is not None else None
    pairs = at.sum(1, keepdim=True).to(f)
    for h in range(H):
        g = h // r
        q, k, x = Q[:, h], K[:, g], V[:, g]
        s = torch.zeros(m, n, dtype=f)
        raw = q.nan_to_num(0, 0, 0) @ k.nan_to_num(0, 0, 0).t()
        s = torch.where(at, torch.where(torch.isfinite(k).all(1)[None, :] & torch.isfinite(q).all(1)[:, None], raw, (q @ k.t())), raw) * p.scale
        if bucket is not None:
            s = s + p.bias.to(f)[:, h][bucket]
        s = s.masked_fill(~at, float("-inf"))
        there = at & (s != float("-inf"))
        L = torch.logsumexp(s, 1, keepdim=True) if n else torch.full((m, 1), float("-inf"), dtype=f)
        L0 = torch.where(L == float("-inf"), torch.zeros_like(L), L)
        P = torch.where(there, torch.exp(s - L0), torch.zeros_like(s))
        s0 = torch.where(there, s, torch.zeros_like(s)).nan_to_num(0, 0, 0)
        es = (D + 8) * v * abs(p.scale) * (q.nan_to_num(0, 0, 0).abs() @ k.nan_to_num(0, 0, 0).abs().t()) + 4 * v * s0.abs()
        e_row = torch.where(there & (s > L - 200), es, torch.zeros_like(es)).amax(1, keepdim=True) if n else torch.zeros(m, 1, dtype=f)
        ep = 2 * e_row + (pairs + 8) * v + (L0.abs().nan_to_num(0, 0, 0) + 2) * 2 * v              # of a weight, relative

        def masked(a, b):                                # a @ b over the attended pairs only
            bad = ~torch.isfinite(b).all(1)
            y = a[:, ~bad] @ b[~bad]
            for j in bad.nonzero().flatten().tolist():
                hit = there[:, j] if a.shape[0] == m else there[j]
                y[hit] += a[hit, j][:, None] * b[j][None, :]
            return y
        O = masked(P, x)
        size = P.abs() @ x.nan_to_num(0, 0, 0).abs()
        out["O"][:, h], out["lse"][h] = O, L[:, 0]
        tol["O"][:, h] = (w16 + ep + (pairs + 8) * v) * size + u * O.abs() + tiny
        tol["lse"][h] = (2 * e_row + (pairs + 8) * v + 4 * v * L0.abs().nan_to_num(0, 0, 0) + 4 * v)[:, 0]
        if not grads:
            continue
        go = dO[:, h]
        dp = go @ x.t()
        delta = (go * O).sum(1, keepdim=True)
        ds = torch.where(there, P * (dp - delta), torch.zeros_like(P))
        e_ds = P * (ep * (dp.abs() + delta.abs()) + (D + 8) * v * (go.abs() @ x.abs().t()) + (u + (D + 8) * v) * (go.abs() * O.abs()).sum(1, keepdim=True)
                    + (go.abs() * (tol["O"][:, h] - u * O.abs())).sum(1, keepdim=True))
        e_op = e_ds + w16 * (ds.abs() + e_ds) + (tiny if w16 else 0) * there
        cols = at.sum(0).to(f)[:, None] * r
        out["dQ"][:, h] = p.scale * (ds @ k)
        tol["dQ"][:, h] = abs(p.scale) * (e_op @ k.abs() + (pairs + 8) * v * (ds.abs() @ k.abs())) + u * out["dQ"][:, h].abs() + tiny
        out["dK"][:, g] += p.scale * (ds.t() @ q)
        tol["dK"][:, g] += abs(p.scale) * (e_op.t() @ q.abs() + (cols + 8) * v * (ds.abs().t() @ q.abs()))
        out["dV"][:, g] += P.t() @ go
        tol["dV"][:, g] += ((w16 + ep) * P + (tiny if w16 else 0) * there).t() @ go.abs() + (cols + 8) * v * (P.t() @ go.abs())
        if bucket is not None:
            out["dT"][:, h] = torch.bincount(bucket.reshape(-1), ds.reshape(-1), minlength=p.bias.shape[0])
            terms = torch.bincount(bucket.reshape(-1), (e_ds + (at.sum() + 8) * v * ds.abs()).reshape(-1), minlength=p.bias.shape[0])
            tol["dT"][:, h] = terms + u * out["dT"][:, h].abs() + tiny
    if grads:
        for k in ("dK", "dV"):
            tol[k] += u * out[k].abs() + tiny
    return {k: (out[k], tol[k]) for k in out}
