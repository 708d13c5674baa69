"""Chunk batches over paged caches, and the operators of include/respec_prompt.h in 64 bits.

Everything is built and evaluated on the host; the tests copy the inputs to the GPU.
"""
import math
from dataclasses import dataclass, field

import torch

F64 = torch.float64


@dataclass
class Chunk:
    """Inputs of one chunk batch, and (k_rows, v_rows)[b]: the cache rows of each sequence in order."""
    dtype: torch.dtype
    heads: int
    kv_heads: int
    head_dim: int
    page: int
    sizes: list                   # (new tokens, rows in front) of each sequence
    q: torch.Tensor               # [T][Hq][D]
    k_new: torch.Tensor           # [T][Hkv][D]
    v_new: torch.Tensor
    k_pages: torch.Tensor         # [pages][Hkv][page][D]; new tokens' rows are written
    v_pages: torch.Tensor
    table: torch.Tensor
    off: torch.Tensor
    kv_len: torch.Tensor
    rows: list = field(default_factory=list)

    @property
    def max_new(self):
        return max([n for n, _ in self.sizes] + [0])

    @property
    def max_kv(self):
        return max([l for _, l in self.sizes] + [0])


def make(sizes, *, dtype=torch.bfloat16, heads=8, kv_heads=2, head_dim=64, page=16, seed=0, stale=math.nan, q_std=2.0,
         spare=2):
    gen = torch.Generator().manual_seed(1000 + seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen) * std).to(dtype)

    total = sum(n for n, _ in sizes)
    pages = [max(-(-(n + l) // page), 0) for n, l in sizes]
    width = max(pages + [1]) + spare
    ids = torch.randperm(sum(pages) + 3, generator=gen).tolist()
    k = torch.full((len(ids), kv_heads, page, head_dim), stale, dtype=dtype)
    v = torch.full_like(k, stale)
    table = torch.full((len(sizes), width), -1, dtype=torch.int32)
    k_new, v_new = normal(total, kv_heads, head_dim), normal(total, kv_heads, head_dim)
    rows, at, t = [], 0, 0
    for b, (n, l) in enumerate(sizes):
        table[b, :pages[b]] = torch.tensor(ids[at:at + pages[b]], dtype=torch.int32)
        at += pages[b]
        kr = torch.cat([normal(l, kv_heads, head_dim), k_new[t:t + n]])
        vr = torch.cat([normal(l, kv_heads, head_dim), v_new[t:t + n]])
        for r in range(n + l):
            k[table[b, r // page], :, r % page] = kr[r]
            v[table[b, r // page], :, r % page] = vr[r]
        rows.append((kr, vr))
        t += n
    off = torch.tensor([0] + [n for n, _ in sizes]).cumsum(0).int()
    return Chunk(dtype, heads, kv_heads, head_dim, page, list(sizes), normal(total, heads, head_dim, std=q_std), k_new,
                 v_new, k, v, table, off, torch.tensor([l for _, l in sizes], dtype=torch.int32), rows)


def attention(c: Chunk, scale=None):
    """(out, tolerance) [T][Hq][D] in 64 bits.

    The tolerance bounds a kernel that takes the products in float32, rounds the weights to the
    workload type before the second product (not for float32), and the result once.  With u the
    type's half step and e = 2^-24: a score is off by at most (D + 4) e sum |q k| scale from its sum
    of D products, its factor and its use in base 2; its weight by twice that (the maximum's own score is in
    it, too), by 2^-22 for exp2, and by u; the sums over the rows add (rows + 64) e at most.  A
    value's share of the output moves with its weight, so the output by sum p |v| times all that,
    plus its own rounding.
    """
    scale = 1 / math.sqrt(c.head_dim) if scale is None else scale
    u = torch.finfo(c.dtype).eps / 2
    e = 2.0 ** -24
    g = c.heads // c.kv_heads
    out = torch.empty(c.q.shape, dtype=F64)
    tol = torch.empty(c.q.shape, dtype=F64)
    t = 0
    for (n, l), (kr, vr) in zip(c.sizes, c.rows):
        if n == 0:
            continue
        kr, vr = kr.to(F64), vr.to(F64)
        sees = torch.arange(n + l)[None] <= l + torch.arange(n)[:, None]
        for h in range(c.heads):
            k, v, q = kr[:, h // g], vr[:, h // g], c.q[t:t + n, h].to(F64)
            z = torch.where(sees, q @ k.T * scale, -math.inf)
            p = torch.softmax(z, 1)
            p = torch.where(sees, p, 0.0)
            size = torch.where(sees, q.abs() @ k.abs().T * scale, 0.0).amax(1, keepdim=True)
            if bool(v.isfinite().all()):
                o, a = p @ v, p @ v.abs()
            else:  # what a token does not see has no part in its output
                pv = torch.where(sees[:, :, None], p[:, :, None] * v[None], 0.0)
                o, a = pv.sum(1), pv.abs().sum(1)
            d = 2 * (c.head_dim + 4) * e * size + 2 ** -22 + (n + l + 64) * e + (u if c.dtype != torch.float32 else 0)
            out[t:t + n, h] = o
            tol[t:t + n, h] = a * d + o.abs() * u + 1e-30
        t += n
    return out, tol


def score(z, token, topk):
    """({output: values}, {output: tolerance}) of respec_score for logits [R][V] (CPU) in 64 bits;
    whole numbers are exact and have no tolerance.

    With e = 2^-24 and d = z - max z: a term e^d is off by 2 |d| e (the difference and its product with log2 e) and
    2^-22 (exp2), a sum by one e for each of the (V / 256 + 16) terms and partial sums that a value goes through, and 8
    for the rescalings: S by s = (2 E|d| + 4 + V / 256 + 24) e of itself, and so log S absolutely.  T / S moves
    by |T / S| times twice that (both sums) and 2 E[d^2] e.  Differences, sums and logarithms add a rounding, e of
    their value, each.
    """
    e = 2.0 ** -24
    zd = z.to(F64)
    vocab = z.shape[1]
    bad = zd.isnan().any(1) | (zd == math.inf).any(1)
    none = (zd == -math.inf).all(1)
    ok = (~bad & ~none)[:, None]
    safe = torch.where(ok, zd, 0.0)
    m = safe.amax(1, keepdim=True)
    d = safe - m
    log_s = d.exp().sum(1, keepdim=True).log()   # (not from lse: rows of the type's lowest value)
    lse, logp = m + log_s, d - log_s
    p, log_s = logp.exp(), log_s[:, 0]
    d = torch.where(p > 0, d, 0.0)
    mean, square = (p * d).sum(1).abs(), (p * d * d).sum(1)
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    ids = torch.arange(vocab)
    order = torch.argsort(torch.where(zd.isnan(), 0.0, zd), dim=1, descending=True, stable=True)[:, :topk]
    tok = token.long().clamp(0, vocab - 1)[:, None]
    valid = (token >= 0) & (token < vocab)
    zt = zd.gather(1, tok)
    rank = ((zd > zt) | ((zd == zt) & (ids < tok))).sum(1)
    lp = logp.gather(1, tok)[:, 0]
    nan, inf = math.nan, math.inf
    lp = torch.where(none, -inf, lp)
    lp = torch.where(token == -1, 0.0, torch.where(valid, lp, nan))
    top = torch.where(none[:, None], -inf, logp.gather(1, order))
    want = {"lse": torch.where(bad, nan, torch.where(none, -inf, lse[:, 0])),
            "entropy": torch.where(bad, nan, torch.where(none, 0.0, entropy)),
            "tok_logprob": torch.where(bad, nan, lp), "tok_rank": torch.where(bad | ~valid, -1, rank).int(),
            "topk_id": torch.where(bad[:, None], -1, order).int(), "topk_logprob": torch.where(bad[:, None], nan, top)}
    s = (2 * mean + 4 + vocab / 256 + 24) * e + log_s * e
    tol = {"lse": s + lse[:, 0].abs() * e, "entropy": s + mean * 2 * s + 2 * square * e + (mean + entropy) * e,
           "tok_logprob": s + 2 * (lp.abs() + log_s) * e,
           "topk_logprob": s[:, None] + 2 * (top.abs() + log_s[:, None]) * e}
    return want, {k: torch.where(v.isfinite(), v, 0.0) + 1e-30 for k, v in tol.items()}
