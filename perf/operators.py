"""What is timed of the prompt side: a paged cache is filled, attended to and the prompt scored.

  append   keys and values of new tokens go into the rows of a paged cache (``ChunkPlan.append``)
  attend   new tokens attend, causally, to their sequence's rows of that cache (``ChunkPlan.attend``)
  score    log probabilities, ranks, entropies and top alternatives of given tokens (``ScorePlan.score``)

A case of append and attend:

  dtype, heads, kv_heads, head_dim   the model's shape
  page                               rows per page; 0: one page per sequence (the cache of a verification step)
  batch                              sequences in the call
  new_min, new_max                   new tokens per sequence (spread over their logarithm)
  len_min, len_max                   rows already in the cache (spread over their logarithm; 0 and 0: whole prompts)
  fused                              q, k and v are slices of one projection's output

A case of score: dtype, vocab, rows, topk, and pad, the unused columns behind each row of logits.

Values: keys and values are N(0, 1), queries N(0, 2.5^2), so that a token attends to some tens of
rows and not to all alike; rows behind a sequence's end hold what a reused page holds (NaN in places), and
the table's entries behind its last page are -1.  Logits are N(0, 2.5^2) with a few peaks; the
scored tokens are drawn from the distributions themselves.
"""
import functools
import math
import random

import torch

own = False

_7B = dict(dtype="bf16", heads=32, kv_heads=32, head_dim=128)
_8B = dict(dtype="bf16", heads=32, kv_heads=8, head_dim=128)
_G7 = dict(dtype="bf16", heads=28, kv_heads=4, head_dim=128)
_D64 = dict(dtype="bf16", heads=32, kv_heads=8, head_dim=64)
_F32 = dict(dtype="f32", heads=4, kv_heads=4, head_dim=64)
_F32_MID = dict(dtype="f32", heads=16, kv_heads=16, head_dim=64)


def _cache_case(op, name, model, batch, new, lens, page, fused=False):
    c = dict(model, op=op, batch=batch, new_min=new[0], new_max=new[1], len_min=lens[0], len_max=lens[1], page=page,
             fused=fused)
    return dict(c, name=name) if name else c


_attend = functools.partial(_cache_case, "attend")
_append = functools.partial(_cache_case, "append")


def _score(name, dtype, rows, vocab, topk, pad=0):
    c = dict(op="score", dtype=dtype, rows=rows, vocab=vocab, topk=topk, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decoding step of a serving batch: one row per sequence and head (launches and latency)
        _append("append-96x1", _8B, 96, (1, 1), (100, 1500), 16),
        # prompts of several requests at once, on a target without grouped heads
        _append("append-prompts", _7B, 5, (300, 4001), (0, 0), 64, fused=True),
        # the smallest call: one token of a small float32 target
        _attend("decode-f32", _F32, 1, (1, 1), (512, 512), 16),
        # one token each of a ragged serving batch
        _attend("decode-batch32", _8B, 32, (1, 1), (300, 16000), 16),
        # one token of one long conversation, groups of seven heads
        _attend("decode-long", _G7, 1, (1, 1), (32767, 32767), 64),
        # a long document goes in piece by piece: one piece over what is there already
        _attend("chunk512-over-16k", _8B, 1, (512, 512), (16384, 16384), 64, fused=True),
        # a whole prompt into the cache of a verification step
        _attend("prompt-8k", _7B, 1, (8192, 8192), (0, 0), 0),
        # prompts, continuations and decoding tokens in one call; odd pages, heads of 64 columns
        _attend("mixed-batch12", _D64, 12, (1, 700), (33, 9000), 24),
        # a prompt of a small float32 target
        _attend("prompt-f32", _F32_MID, 1, (1500, 1500), (0, 0), 16),
        # one row: the entropy and alternatives of a single decoding step
        _score("score-1", "f32", 1, 32000, 8),
        # the nodes of a full draft tree on a target with a large vocabulary
        _score("score-tree65", "f32", 65, 152064, 16),
        # a chunk of a prompt, logits as a bf16 product leaves them, padded rows
        _score("score-prompt2k", "bf16", 2048, 128256, 8, pad=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_LARGEST = 32 * 8192 * 8192   # scores of the largest listed case, as the plain form holds them


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "chunk", "prompt", "mixed", "f32", "score", "score"])
    if kind == "score":
        dtype, vocab = rng.choice(["f32", "bf16"]), _log(rng, 3000, 152064)
        rows = _log(rng, 1, max(1, min(4096, 260_000_000 // vocab)))
        return _score("", dtype, rows, vocab, rng.choice([1, 5, 8, 16]), rng.choice([0, 0, 8, 64]))
    model = rng.choice([_7B, _8B, _G7, _D64])
    page = rng.choice([16, 16, 24, 64, 128, 0])
    if kind == "append":
        b = _log(rng, 1, 64)
        top = _log(rng, 1, max(1, 8192 // b))
        length = rng.choice([0, _log(rng, 10, 2000)])
        model = rng.choice([model, _F32_MID])
        return _append("", model, b, (rng.randint(1, top), top), (length // 3, length), page, rng.random() < 0.5)
    if kind == "decode":
        b = _log(rng, 1, 64)
        longest = _log(rng, 64, min(32768, 500_000 // b))
        top = rng.choice([1, 1, 1, 4])
        return _attend("", model, b, (1, top), (_log(rng, 16, longest), longest), page, rng.random() < 0.5)
    if kind == "chunk":
        n, length = _log(rng, 16, 1024), _log(rng, 64, 32768)
        return _attend("", model, 1, (n, n), (length, length), page, rng.random() < 0.5)
    if kind == "prompt":
        b = rng.randint(1, 6)
        top = _log(rng, 64, 8192 // b)
        return _attend("", model, b, (_log(rng, 16, top), top), (0, 0), page, rng.random() < 0.5)
    if kind == "mixed":
        b = rng.randint(2, 16)
        longest = _log(rng, 200, 9000)
        top = _log(rng, 16, min(700, _LARGEST // (32 * b * longest)))
        return _attend("", model, b, (1, top), (_log(rng, 16, longest), longest), page, rng.random() < 0.5)
    model = dict(rng.choice([_F32, _F32_MID]), head_dim=rng.choice([64, 128]))
    n, length = _log(rng, 1, 1500), rng.choice([0, _log(rng, 16, 2000)])
    return _attend("", model, 1, (n, n), (length, length), page)


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _sizes(case):
    """(new tokens, rows in the cache) of every sequence; the same set for every seed."""
    def spread(lo, hi):
        b = case["batch"]
        if lo == hi or b == 1:
            return [hi] * b
        a, z = math.log(max(lo, 1)), math.log(hi)
        return [int(round(math.exp(a + i / (b - 1) * (z - a)))) for i in range(b)]

    news, lens = spread(case["new_min"], case["new_max"]), spread(case["len_min"], case["len_max"])
    random.Random(case["batch"]).shuffle(news)
    return list(zip(news, lens))


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        # the logits once; per logit a difference, an exponential, two sums, a maximum and the rank's comparisons
        return {"bytes": rows * vocab * es + rows * (4 + 16 + 8 * case["topk"]), "flops": 10 * rows * vocab}
    sizes, d = _sizes(case), case["head_dim"]
    tokens, row = sum(n for n, _ in sizes), 2 * case["kv_heads"] * d * es
    if case["op"] == "append":
        return {"bytes": 2 * tokens * row, "flops": 0}
    return {"bytes": 2 * tokens * case["heads"] * d * es + sum((n + l) * row for n, l in sizes),
            "flops": sum(4 * case["heads"] * d * (n * l + n * (n + 1) // 2) for n, l in sizes)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _cache_inputs(case, seed):
    dev, dt = torch.device("cuda"), _dtype(case)
    rng = random.Random(seed * 1000003 + 29)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    sizes = _sizes(case)
    rng.shuffle(sizes)
    b, d, h, hkv = case["batch"], case["head_dim"], case["heads"], case["kv_heads"]
    tokens = sum(n for n, _ in sizes)
    longest = max(n + l for n, l in sizes)
    page = case["page"] or -(-(longest + 64) // 64) * 64
    pages = [-(-(n + l) // page) for n, l in sizes]
    width, total = max(pages) + 2, sum(pages) + 3

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dt, device=dev).normal_(0.0, std, generator=gen)

    ints = functools.partial(torch.tensor, dtype=torch.int32, device=dev)
    ids = list(range(total))
    if case["page"]:
        rng.shuffle(ids)
    table, at = [], 0
    for n in pages:
        table.append(ids[at:at + n] + [-1] * (width - n))
        at += n
    off = [0]
    for n, _ in sizes:
        off.append(off[-1] + n)
    k, v = normal(total, hkv, page, d), normal(total, hkv, page, d)
    if case["op"] == "attend":  # what was never a row of these sequences
        for (n, l), row in zip(sizes, table):
            last = n + l - 1
            k[row[last // page], :, last % page + 1:] = math.nan
            v[row[last // page], :, last % page + 1:] = math.nan
    if case["fused"]:
        qkv = normal(tokens, h + 2 * hkv, d)
        q, k_new, v_new = qkv[:, :h], qkv[:, h:h + hkv], qkv[:, h + hkv:]
        q *= 2.5
    else:
        q, k_new, v_new = normal(tokens, h, d, std=2.5), normal(tokens, hkv, d), normal(tokens, hkv, d)
    return dict(q=q, k_new=k_new, v_new=v_new, k_pages=k, v_pages=v, page_table=ints(table), new_off=ints(off),
                kv_len=ints([l for _, l in sizes])), sizes


def _score_inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    z = torch.empty(rows, vocab + case["pad"], dtype=torch.float32, device=dev).normal_(0.0, 2.5, generator=gen)
    peaks = torch.randint(vocab, (rows, 6), generator=gen, device=dev)
    z.scatter_add_(1, peaks, torch.rand(rows, 6, generator=gen, device=dev) * 16)
    z = z.to(_dtype(case))[:, :vocab]
    # a sample of each row's distribution: the largest of z + Gumbel noise
    token = torch.empty(rows, dtype=torch.int32, device=dev)
    for lo in range(0, rows, 256):
        u = torch.empty(z[lo:lo + 256].shape, device=dev).exponential_(generator=gen)
        token[lo:lo + 256] = (z[lo:lo + 256].float() - u.log()).argmax(1).int()
    return dict(logits=z, token=token)


def prepare(case, seed):
    if case["op"] == "score":
        s = dict(_score_inputs(case, seed), case=case)
        if own:
            from paper_2511_01282_amd import binding, prompt
            s["plan"] = prompt.ScorePlan(vocab=case["vocab"], max_rows=case["rows"], topk_out=case["topk"],
                                         dtype=binding.F32 if case["dtype"] == "f32" else binding.BF16)
            s["out"] = prompt.alloc_score_outputs(rows=case["rows"], topk_out=case["topk"])
        return s
    s, sizes = _cache_inputs(case, seed)
    s["case"] = case
    s["sizes"] = dict(max_new_in_batch=max(n for n, _ in sizes), max_kv_len_in_batch=max(l for _, l in sizes))
    s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=s["q"].device)
    if own:
        from paper_2511_01282_amd import binding, prompt
        s["plan"] = prompt.ChunkPlan(n_q_heads=case["heads"], n_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                                     dtype=binding.F32 if case["dtype"] == "f32" else binding.BF16,
                                     max_batch=case["batch"], max_new=len(s["q"]),
                                     max_kv_len=s["sizes"]["max_kv_len_in_batch"])
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _plain_append(s):
    table, off, page = s["page_table"].long(), s["new_off"].long(), s["k_pages"].shape[2]
    t = torch.arange(len(s["k_new"]), device=off.device)
    b = torch.searchsorted(off[1:].contiguous(), t, right=True)
    row = s["kv_len"].long()[b] + t - off[b]
    at = table[b, row // page]
    s["k_pages"][at, :, row % page] = s["k_new"]
    s["v_pages"][at, :, row % page] = s["v_new"]
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attend(s):
    table, off, kv_len = s["page_table"].long(), s["new_off"].long(), s["kv_len"].long()
    q, page = s["q"], s["k_pages"].shape[2]
    tokens, h, d = q.shape
    b, hkv = len(kv_len), s["k_pages"].shape[1]
    n, rows = s["sizes"]["max_new_in_batch"], s["sizes"]["max_new_in_batch"] + s["sizes"]["max_kv_len_in_batch"]
    # every sequence padded to the longest: rows of the cache, then tokens
    pos = torch.arange(rows, device=q.device)
    new = off[1:] - off[:-1]
    here = pos[None] < (kv_len + new)[:, None]
    at = table[:, (pos // page).clamp(max=table.shape[1] - 1)].clamp(min=0)
    k = torch.where(here[:, :, None, None], s["k_pages"][at, :, pos % page].float(), 0.0)
    v = torch.where(here[:, :, None, None], s["v_pages"][at, :, pos % page].float(), 0.0)
    i = torch.arange(n, device=q.device)
    live = i[None] < new[:, None]
    tok = torch.where(live, off[:-1, None] + i, tokens)
    g = h // hkv
    qp = q[tok.clamp(max=tokens - 1)].float().reshape(b, n, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * n, d)
    z = torch.matmul(qp, k.permute(0, 2, 3, 1).contiguous()).mul_(1 / math.sqrt(d)).view(b, hkv, g, n, rows)
    sees = pos[None, None] <= kv_len[:, None, None] + i[None, :, None]
    z.masked_fill_(~sees[:, None, None], -math.inf)
    p = z.sub_(z.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p.view(b, hkv, g * n, rows), v.permute(0, 2, 1, 3).contiguous())
    o = o.view(b, hkv, g, n, d) / p.sum(-1, keepdim=True)
    out = torch.empty(tokens + 1, h, d, dtype=q.dtype, device=q.device)
    out[tok] = o.permute(0, 3, 1, 2, 4).reshape(b, n, h, d).to(q.dtype)
    return out[:tokens]


def _plain_score(s):
    z, token, k = s["logits"].float(), s["token"].long()[:, None], s["case"]["topk"]
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    entropy = log_total - (e * (z - m)).sum(1, keepdim=True) / total
    zt = z.gather(1, token)
    ids = torch.arange(z.shape[1], device=z.device)
    rank = ((z > zt) | ((z == zt) & (ids < token))).sum(1)
    # the k largest by (value, lowest id): one 64-bit key that orders both
    bits = torch.where(z == 0, 0.0, z).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    top = ((order << 32) + (0x7FFFFFFF - ids)).topk(k, 1).values
    top = 0x7FFFFFFF - (top & 0xFFFFFFFF)
    return {"tok_logprob": (zt - m - log_total)[:, 0], "tok_rank": rank.int(), "lse": (m + log_total)[:, 0],
            "entropy": entropy[:, 0], "topk_id": top.int(), "topk_logprob": z.gather(1, top) - m - log_total}


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "score": _plain_score}[op](s)
    if op == "score":
        s["plan"].score(s["logits"], s["token"], s["out"])
        return s["out"]
    if op == "append":
        s["plan"].append(s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["page_table"], s["new_off"], s["kv_len"],
                         max_new_in_batch=s["sizes"]["max_new_in_batch"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    s["plan"].attend(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["new_off"], s["kv_len"], s["out"],
                     **s["sizes"])
    return s["out"]


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    f64 = torch.float64
    if case["op"] == "score":
        s = _score_inputs(case, seed)
        outs = {"tok_logprob": [], "lse": [], "entropy": [], "topk_logprob": []}
        for lo in range(0, case["rows"], 128):
            z = s["logits"][lo:lo + 128].to(f64)
            lse = torch.logsumexp(z, 1)
            logp = z - lse[:, None]
            outs["lse"].append(lse)
            outs["tok_logprob"].append(logp.gather(1, s["token"][lo:lo + 128, None].long())[:, 0])
            outs["entropy"].append(-(logp.exp() * logp).sum(1))
            outs["topk_logprob"].append(logp.topk(case["topk"], 1).values)
        return dict({k: torch.cat(v) for k, v in outs.items()}, tok_rank=None, topk_id=None)
    s, sizes = _cache_inputs(case, seed)
    table, page, at = s["page_table"].tolist(), s["k_pages"].shape[2], 0
    if case["op"] == "append":
        for (n, length), pages in zip(sizes, table):
            done = 0
            while done < n:
                r = length + done
                c = min(n - done, page - r % page)
                for to, new in ((s["k_pages"], s["k_new"]), (s["v_pages"], s["v_new"])):
                    to[pages[r // page], :, r % page:r % page + c] = new[at + done:at + done + c].transpose(0, 1)
                done += c
            at += n
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    h, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.empty(s["q"].shape, dtype=f64, device=s["q"].device)
    for (n, length), pages in zip(sizes, table):
        rows = length + n
        used = pages[:-(-rows // page)]
        for c in range(hkv):
            k = s["k_pages"][used, c].reshape(-1, d)[:rows].to(f64)
            v = s["v_pages"][used, c].reshape(-1, d)[:rows].to(f64)
            for j in range(c * h // hkv, (c + 1) * h // hkv):
                for lo in range(0, n, 2048):
                    hi = min(n, lo + 2048)
                    a = s["q"][at + lo:at + hi, j].to(f64) @ k.t().contiguous() / math.sqrt(d)
                    i = torch.arange(lo, hi, device=a.device)[:, None]
                    a.masked_fill_(torch.arange(rows, device=a.device)[None] > length + i, -math.inf)
                    out[at + lo:at + hi, j] = torch.softmax(a, 1) @ v
        at += n
    return out
