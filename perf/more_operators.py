"""What is timed of a cache's life around the steps: rotary positions, a cache of 8-bit values, rows kept, pages copied.

  rotary   queries and keys of new tokens, or of the nodes of a draft tree, are turned to their positions
           (``cache.RotaryPlan.rotate``)
  append   keys and values of new tokens go into a paged cache of e4m3 values with a power-of-two scale for each block of
           rows and head (``ChunkPlan.append_q8``)
  attend   new tokens attend, causally, to their sequence's rows of that cache (``ChunkPlan.attend_q8``)
  keep     the accepted path of every verified draft tree moves to the front of its nodes' rows, in all layers
           (``cache.CacheLayers.keep_rows``)
  copy     pages are copied: the partly filled ones of forked sequences, or the pages of beams (``cache.CacheLayers.copy_pages``)

Cases: dtype, heads, kv_heads, head_dim are the model's shape, page the rows of a page (0: one page per sequence), block the
rows that share a scale.  rotary: tokens of ``batch`` sequences (0: positions are given one by one, as for a tree),
``far``, the largest position, rotary_dim and layout, and fused: q and k are slices of one projection's output.  append and
attend: new tokens (new_min .. new_max) and rows that are there already (len_min .. len_max) per sequence, spread over
their logarithm.  keep: nodes per tree, the longest accepted path, layers.  copy: pages of the pool, pairs, layers, and
``eight``: a cache of 8-bit values with its scales.

Values: keys and values are N(0, a^2) with an ``a`` of each page and head, queries N(0, 2.5^2); rows behind a
sequence's end hold what a reused page holds, NaN in places, and the table's entries behind its last page are -1.
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


def _named(name, c):
    return dict(c, name=name) if name else c


def _rotary(name, model, tokens, batch, far, rotary_dim, layout, fused=False):
    return _named(name, dict(model, op="rotary", tokens=tokens, batch=batch, far=far, rotary_dim=rotary_dim, layout=layout,
                             fused=fused))


def _cache_case(op, name, model, batch, new, lens, page, block, fused=False):
    return _named(name, dict(model, op=op, batch=batch, new_min=new[0], new_max=new[1], len_min=lens[0], len_max=lens[1],
                             page=page, block=block, fused=fused))


_append = functools.partial(_cache_case, "append")
_attend = functools.partial(_cache_case, "attend")


def _keep(name, model, layers, batch, nodes, longest, lens, page):
    return _named(name, dict(model, op="keep", layers=layers, batch=batch, nodes=nodes, longest=longest, len_min=lens[0],
                             len_max=lens[1], page=page))


def _copy(name, model, layers, pages, pairs, page, block, eight):
    return _named(name, dict(model, op="copy", layers=layers, pages=pages, pairs=pairs, page=page, block=block, eight=eight))


def listed():
    return [
        # the nodes of a full draft tree deep in a long conversation (launches and latency)
        _rotary("rotary-tree65", _G7, 65, 0, 131072, 128, "half"),
        # prompts of four requests, as slices of one projection
        _rotary("rotary-prompts", _8B, 8192, 4, 9000, 128, "half", fused=True),
        # a decoding step of a serving batch: one row per sequence and head
        _append("append-96x1", _8B, 96, (1, 1), (100, 1500), 16, 16),
        # prompts of several requests at once, on a target without grouped heads
        _append("append-prompts", _7B, 5, (300, 4001), (0, 0), 64, 32, fused=True),
        # one token each of a ragged serving batch
        _attend("decode-batch32", _8B, 32, (1, 1), (300, 16000), 16, 16),
        # one token of one long conversation, groups of seven heads
        _attend("decode-long", _G7, 1, (1, 1), (32767, 32767), 64, 64),
        # a long document goes in piece by piece: one piece over what is there already
        _attend("chunk512-over-16k", _8B, 1, (512, 512), (16384, 16384), 64, 32, fused=True),
        # prompts, continuations and decoding tokens in one call; heads of 64 columns, pages that end inside tiles
        _attend("mixed-batch12", _D64, 12, (1, 700), (33, 9000), 48, 16),
        # after a verification step of one sequence: its path, in the caches of all layers
        _keep("keep-tree26", _7B, 32, 1, 26, 5, (200, 200), 0),
        # after a step of a batch with full trees, paged caches
        _keep("keep-batch8x65", _8B, 32, 8, 65, 12, (100, 900), 64),
        # four samples go on from one prompt: its last page, 8-bit values and scales
        _copy("fork-4", _8B, 32, 64, 4, 16, 16, True),
        # beams take over each other's pages
        _copy("copy-24-pages", _8B, 32, 64, 24, 64, 0, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_LARGEST = 32 * 512 * 16896   # scores of the largest listed case, as the plain form holds them


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "append", "append", "decode", "decode", "chunk", "prompt", "mixed", "f32", "keep",
                       "keep", "copy", "copy"])
    model = rng.choice([_7B, _8B, _G7, _D64])
    if kind == "rotary":
        model = rng.choice([model, _F32, _F32_MID])
        tokens = _log(rng, 1, 8192)
        if model["dtype"] == "f32" or model is _7B:
            tokens = min(tokens, 4096)
        batch = rng.choice([0, min(tokens, rng.randint(1, 6))])
        return _rotary("", model, tokens, batch, max(tokens, _log(rng, 100, 1_000_000)),
                       model["head_dim"] // rng.choice([1, 1, 2, 4]), rng.choice(["half", "interleaved"]), rng.random() < 0.5)
    block = rng.choice([16, 16, 32, 64, 128])
    page = rng.choice([0, block, block, 2 * block, 3 * block])
    if kind == "append":
        b = _log(rng, 1, 64)
        top = _log(rng, 1, max(1, 8000 // b))
        length = rng.choice([0, _log(rng, 10, 2000)])
        model = rng.choice([model, _F32_MID])
        return _append("", model, b, (rng.randint(1, top), top), (length // 3, length), page, block, rng.random() < 0.5)
    if kind == "decode":
        b = _log(rng, 1, 64)
        longest = _log(rng, 64, min(32768, 300_000 // b))
        top = rng.choice([1, 1, 1, 4])
        return _attend("", model, b, (1, top), (_log(rng, 16, longest), longest), page, block, rng.random() < 0.5)
    if kind == "chunk":
        n, length = _log(rng, 16, 512), _log(rng, 64, 16384)
        return _attend("", model, 1, (n, n), (length, length), page, block, rng.random() < 0.5)
    if kind == "prompt":
        b = rng.randint(1, 6)
        top = _log(rng, 64, int((_LARGEST / (32 * b)) ** 0.5))
        return _attend("", model, b, (_log(rng, 16, top), top), (0, 0), page, block, rng.random() < 0.5)
    if kind == "mixed":
        b = rng.randint(2, 16)
        longest = _log(rng, 200, 9000)
        top = _log(rng, 16, max(16, min(700, _LARGEST // (32 * b * longest))))
        return _attend("", model, b, (1, top), (_log(rng, 16, longest), longest), page, block, rng.random() < 0.5)
    if kind == "f32":
        model = dict(rng.choice([_F32, _F32_MID]), head_dim=rng.choice([64, 128]))
        n, length = _log(rng, 1, 1000), rng.choice([0, _log(rng, 16, 2000)])
        return _attend("", model, 1, (n, n), (length, length), page, block)
    if kind == "keep":
        model = rng.choice([model, _F32_MID])
        b, nodes = rng.randint(1, 8), rng.randint(4, 65)
        length = _log(rng, 16, 900)
        return _keep("", model, rng.choice([1, 4, 16]), b, nodes, rng.randint(1, min(12, (nodes - 1) // 2)),
                     (max(1, length // 4), length), rng.choice([0, 16, 24, 64]))
    eight = rng.random() < 0.5
    pages = _log(rng, 4, 64)
    return _copy("", model, rng.choice([1, 4, 16]), pages, rng.randint(1, max(1, pages // 2 - 1)), rng.choice([1, 2, 4]) * 16,
                 16 if eight else 0, eight)


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _spread(lo, hi, b):
    if lo == hi or b == 1:
        return [hi] * b
    a, z = math.log(max(lo, 1)), math.log(hi)
    return [int(round(math.exp(a + i / (b - 1) * (z - a)))) for i in range(b)]


def _sizes(case):
    """(new tokens, rows in the cache) of every sequence; the same set for every seed."""
    news = _spread(case["new_min"], case["new_max"], case["batch"])
    random.Random(case["batch"]).shuffle(news)
    return list(zip(news, _spread(case["len_min"], case["len_max"], case["batch"])))


def _accepted(case):
    """Accepted tokens of every tree, from 1 to the longest path; the same set for every seed."""
    return [1 + (case["longest"] - 1 - i) % case["longest"] for i in range(case["batch"])]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def work(case):
    es, d, h, hkv = 4 if case["dtype"] == "f32" else 2, case["head_dim"], case["heads"], case["kv_heads"]
    if case["op"] == "rotary":
        # every row read and written; per pair two sums of two products
        return {"bytes": 2 * case["tokens"] * (h + hkv) * d * es, "flops": 3 * case["tokens"] * (h + hkv) * case["rotary_dim"]}
    if case["op"] == "keep":
        return {"bytes": 4 * sum(_accepted(case)) * case["layers"] * hkv * d * es, "flops": 0}
    if case["op"] == "copy":
        row = d + 1 / case["block"] if case["eight"] else d * es
        return {"bytes": int(4 * case["pairs"] * case["layers"] * hkv * case["page"] * row), "flops": 0}
    sizes = _sizes(case)
    tokens, row = sum(n for n, _ in sizes), 2 * hkv * d
    if case["op"] == "append":
        # per element a maximum, a product and a rounding
        return {"bytes": tokens * row * (es + 1), "flops": 3 * tokens * row}
    return {"bytes": 2 * tokens * h * d * es + sum((n + l) * row * (1 + 1 / (d * case["block"])) for n, l in sizes),
            "flops": sum(4 * h * d * (n * l + n * (n + 1) // 2) for n, l in sizes)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generators(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return random.Random(seed * 1000003 + 29), gen


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(counts):
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    return off


def _table(rng, pages, total, shuffle):
    """Rows of page ids, -1 behind each sequence's last."""
    ids, table, at = list(range(total)), [], 0
    if shuffle:
        rng.shuffle(ids)
    for n in pages:
        table.append(ids[at:at + n] + [-1] * (max(pages) + 2 - n))
        at += n
    return table


def _frequencies(case):
    """Radians per position of every pair of columns: a long context's, the slow ones stretched by 8."""
    f = [500000.0 ** (-2 * i / case["rotary_dim"]) for i in range(case["rotary_dim"] // 2)]
    return [w if 2 * math.pi / w < 2048 else w / 8 for w in f]


def _rotary_inputs(case, seed):
    rng, gen = _generators(seed)
    t, h, hkv, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    x = torch.empty(t, h + 2 * hkv if case["fused"] else h + hkv, d, dtype=_dtype(case), device="cuda").normal_(generator=gen)
    q, k = x[:, :h], x[:, h:h + hkv]
    s = dict(q=q, k=k) if case["fused"] else dict(q=q.contiguous(), k=k.contiguous())
    if case["batch"] == 0:
        first = rng.randint(0, max(0, case["far"] - 64))
        pos = [first + min(rng.randint(0, 1 + i // 4), case["far"] - first) for i in range(t)]
        s.update(positions=_ints(pos))
    else:
        b = case["batch"]
        counts = [t // b + (i < t % b) for i in range(b)]
        lens = [rng.randint(0, case["far"] - n) for n in counts]
        s.update(new_off=_ints(_offsets(counts)), kv_len=_ints(lens))
        pos = [l + i for n, l in zip(counts, lens) for i in range(n)]
    return s, pos


def _power(amax):
    """The exponent of a block's scale: the least k of -126 and up with amax <= 448 2^k."""
    m, e = torch.frexp(amax)
    return torch.where(amax > 0, e - 9 + (m > 0.875), -126).clamp(min=-126)


def _codes(x, k):
    """x as e4m3 values of 2^k (float32 in, e4m3 out); what is not finite is NaN."""
    return torch.where(x.isfinite(), torch.ldexp(x, -k), math.nan).to(torch.float8_e4m3fn)


def _amax(x, dims):
    return torch.where(x.isfinite(), x.abs(), 0.0).amax(dims)


def _cache_inputs(case, seed):
    rng, gen = _generators(seed)
    sizes = _sizes(case)
    rng.shuffle(sizes)
    d, h, hkv, block = case["head_dim"], case["heads"], case["kv_heads"], case["block"]
    tokens = sum(n for n, _ in sizes)
    longest = max(n + l for n, l in sizes)
    page = case["page"] or -(-(longest + 64) // 128) * 128
    pages = [-(-(n + l) // page) for n, l in sizes]
    total = sum(pages) + 3
    table = _table(rng, pages, total, case["page"] > 0)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=_dtype(case), device="cuda").normal_(0.0, std, generator=gen)

    def cache():
        codes = torch.empty(total, hkv, page, d, dtype=torch.float8_e4m3fn, device="cuda")
        scale = torch.empty(total, hkv, page // block, dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 27) // (hkv * page * d))
        for lo in range(0, total, step):
            n = min(step, total - lo)
            x = torch.empty(n, hkv, page // block, block, d, device="cuda").normal_(generator=gen)
            x *= torch.empty(n, hkv, 1, 1, 1, device="cuda").normal_(0.0, 0.25, generator=gen).exp_()
            k = _power(x.abs().amax((3, 4)))
            codes[lo:lo + n] = _codes(x, k[..., None, None]).view(n, hkv, page, d)
            scale[lo:lo + n] = (k + 127).to(torch.uint8)
        return codes, scale.view(torch.float8_e8m0fnu)

    (k, k_scale), (v, v_scale) = cache(), cache()
    if case["op"] == "attend":  # what was never a row of these sequences
        for (n, l), row in zip(sizes, table):
            last = n + l - 1
            for x in (k, v):
                x.view(torch.uint8)[row[last // page], :, last % page + 1:] = 0x7F
    if case["fused"]:
        qkv = normal(tokens, h + 2 * hkv, d)
        q, k_new, v_new = qkv[:, :h], qkv[:, h:h + hkv], qkv[:, h + hkv:]
        q *= 2.5
    else:
        q, k_new, v_new = normal(tokens, h, d, std=2.5), normal(tokens, hkv, d), normal(tokens, hkv, d)
    return dict(q=q, k_new=k_new, v_new=v_new, k_pages=k, v_pages=v, k_scale=k_scale, v_scale=v_scale,
                page_table=_ints(table), new_off=_ints(_offsets(n for n, _ in sizes)), kv_len=_ints([l for _, l in sizes])), sizes


def _keep_inputs(case, seed):
    rng, gen = _generators(seed)
    lens, accepted, nodes = _spread(case["len_min"], case["len_max"], case["batch"]), _accepted(case), case["nodes"]
    rng.shuffle(lens)
    rng.shuffle(accepted)
    page = case["page"] or -(-(max(lens) + nodes) // 64) * 64
    pages = [-(-(l + nodes) // page) for l in lens]
    total = sum(pages) + 2
    table = _table(rng, pages, total, case["page"] > 0)
    # the root, then a chain of nodes behind those that the kept rows take (a second candidate's)
    paths = [[0] + sorted(rng.sample(range(a + 1, nodes), a)) for a in accepted]
    width = case["longest"] + 2
    shape = (case["layers"], total, case["kv_heads"], page, case["head_dim"])
    k, v = (torch.empty(shape, dtype=_dtype(case), device="cuda").normal_(generator=gen) for _ in range(2))
    return dict(k_cache=k, v_cache=v, page_table=_ints(table), kv_len=_ints(lens),
                path=_ints([p + [-1] * (width - len(p)) for p in paths]), acc_len=_ints(accepted),
                kv_len_out=torch.empty(case["batch"], dtype=torch.int32, device="cuda")), paths, lens, table


def _copy_inputs(case, seed):
    rng, gen = _generators(seed)
    ids = list(range(case["pages"]))
    rng.shuffle(ids)
    n = case["pairs"]
    src = [ids[n + rng.randrange(case["pages"] - n)] for _ in range(n)]
    shape = (case["layers"], case["pages"], case["kv_heads"], case["page"], case["head_dim"])

    def plane(shape):
        if not case["eight"]:
            return torch.empty(shape, dtype=_dtype(case), device="cuda").normal_(generator=gen)
        return torch.randint(1, 0x7E, shape, dtype=torch.uint8, generator=gen, device="cuda")

    planes = [plane(shape), plane(shape)]
    if case["eight"]:
        planes = [p.view(torch.float8_e4m3fn) for p in planes]
        planes += [(plane(shape[:3] + (case["page"] // case["block"],)) // 8 + 116).view(torch.float8_e8m0fnu) for _ in range(2)]
    return dict(planes=planes, src=_ints(src), dst=_ints(ids[:n])), src, ids[:n]


def prepare(case, seed):
    if own:
        from paper_2511_01282_amd import binding, cache, prompt
        dtype = binding.F32 if case["dtype"] == "f32" else binding.BF16
    if case["op"] == "rotary":
        s, _ = _rotary_inputs(case, seed)
        s.update(case=case, frequencies=_frequencies(case), q_out=torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda"),
                 k_out=torch.empty(s["k"].shape, dtype=s["k"].dtype, device="cuda"))
        if own:
            s["plan"] = cache.RotaryPlan(n_q_heads=case["heads"], n_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                                         rotary_dim=case["rotary_dim"], dtype=dtype, frequencies=s["frequencies"],
                                         layout=cache.HALF if case["layout"] == "half" else cache.INTERLEAVED)
        return s
    if case["op"] == "keep":
        s = dict(_keep_inputs(case, seed)[0], case=case)
        if own:
            s["layers"] = cache.CacheLayers(s["k_cache"], s["v_cache"])
        return s
    if case["op"] == "copy":
        s = dict(_copy_inputs(case, seed)[0], case=case)
        if own:
            s["layers"] = cache.CacheLayers(*s["planes"])
        return s
    s, sizes = _cache_inputs(case, seed)
    s["case"] = case
    s["sizes"] = dict(max_new_in_batch=max(n for n, _ in sizes), max_kv_len_in_batch=max(l for _, l in sizes))
    s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    if own:
        s["plan"] = prompt.ChunkPlan(n_q_heads=case["heads"], n_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                                     dtype=dtype, max_batch=case["batch"], max_new=len(s["q"]),
                                     max_kv_len=s["sizes"]["max_kv_len_in_batch"])
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _plain_rotary(s):
    q, r, half = s["q"], s["case"]["rotary_dim"], s["case"]["layout"] == "half"
    pos = s.get("positions")
    if pos is None:
        t, off = torch.arange(len(q), device=q.device), s["new_off"].long()
        b = torch.searchsorted(off[1:].contiguous(), t, right=True)
        pos = s["kv_len"].long()[b] + t - off[b]
    angle = pos.double()[:, None] * torch.tensor(s["frequencies"], dtype=torch.float64, device=q.device)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x):
        y = x.float()
        a, b = (y[..., :r // 2], y[..., r // 2:r]) if half else (y[..., :r:2], y[..., 1:r:2])
        pair = (a * cos - b * sin, b * cos + a * sin)
        return torch.cat([torch.cat(pair, -1) if half else torch.stack(pair, -1).flatten(-2), y[..., r:]], -1).to(x.dtype)

    return {"q": turn(q), "k": turn(s["k"])}


def _plain_append(s):
    table, off, kv_len, block = s["page_table"].long(), s["new_off"].long(), s["kv_len"].long(), s["case"]["block"]
    page, n = s["k_pages"].shape[2], s["sizes"]["max_new_in_batch"]
    new = off[1:] - off[:-1]
    # every block that a sequence's new rows touch, padded to the most: [B, U] blocks of [block] rows
    first = kv_len // block
    blk = first[:, None] + torch.arange((n + block - 2) // block + 1, device=off.device)
    row = blk[:, :, None] * block + torch.arange(block, device=off.device)
    live = blk * block < (kv_len + new)[:, None]
    old = row < kv_len[:, None, None]
    fresh = ~old & (row < (kv_len + new)[:, None, None])
    b = torch.arange(len(kv_len), device=off.device)[:, None].expand_as(blk)
    b, blk, row, old, fresh = b[live], blk[live], row[live], old[live], fresh[live]   # [X], [X, block]
    at, sub = table[b, blk * block // page], blk % (page // block)
    tok = torch.where(fresh, off[b, None] + row - kv_len[b, None], 0)
    within = row % page
    for codes, scale, x_new in ((s["k_pages"], s["k_scale"], s["k_new"]), (s["v_pages"], s["v_scale"], s["v_new"])):
        raw, power = codes.view(torch.uint8), scale.view(torch.uint8)
        x = torch.where(fresh[:, :, None, None], x_new[tok].float(), 0.0)                    # [X, block, Hkv, D]
        was = power[at, :, sub].int() - 127                                                      # [X, Hkv]
        k = _power(_amax(x, (1, 3)))
        k = torch.where(old[:, :1], torch.maximum(k, was), k)
        before = raw[at[:, None], :, within]                                                       # [X, block, Hkv, D]
        x = torch.where(old[:, :, None, None], torch.ldexp(before.view(torch.float8_e4m3fn).float(), was[:, None, :, None]), x)
        y = torch.where((old | fresh)[:, :, None, None], _codes(x, k[:, None, :, None]).view(torch.uint8), before)
        raw[at[:, None], :, within] = y
        power[at, :, sub] = (k + 127).to(torch.uint8)
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attend(s):
    table, off, kv_len, block = s["page_table"].long(), s["new_off"].long(), s["kv_len"].long(), s["case"]["block"]
    q, page = s["q"], s["k_pages"].shape[2]
    tokens, h, d = q.shape
    b, hkv = len(kv_len), s["k_pages"].shape[1]
    n, rows = s["sizes"]["max_new_in_batch"], s["sizes"]["max_new_in_batch"] + s["sizes"]["max_kv_len_in_batch"]
    # every sequence padded to the longest: rows of the cache, then tokens
    pos = torch.arange(rows, device=q.device)
    new = off[1:] - off[:-1]
    here = pos[None] < (kv_len + new)[:, None]
    at = table[:, (pos // page).clamp(max=table.shape[1] - 1)].clamp(min=0)

    def values(codes, scale):
        x = codes.view(torch.uint8)[at, :, pos % page].view(torch.float8_e4m3fn).float()
        x = torch.ldexp(x, scale.view(torch.uint8)[at, :, pos % page // block].int()[..., None] - 127)
        return torch.where(here[:, :, None, None], x, 0.0)

    k, v = values(s["k_pages"], s["k_scale"]), values(s["v_pages"], s["v_scale"])
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


def _plain_keep(s):
    table, kv_len, acc, path = s["page_table"].long(), s["kv_len"].long(), s["acc_len"].long(), s["path"].long()
    page, i = s["k_cache"].shape[3], torch.arange(path.shape[1], device=path.device)
    b = torch.arange(len(kv_len), device=path.device)[:, None].expand_as(path)
    live = i <= acc[:, None]
    frm, to = (kv_len[:, None] + path)[live], (kv_len[:, None] + i)[live]
    b = b[live]
    p0, p1 = table[b, frm // page], table[b, to // page]
    for x in (s["k_cache"], s["v_cache"]):
        x[:, p1, :, to % page] = x[:, p0, :, frm % page]
    s["kv_len_out"].copy_(kv_len + acc + 1)
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_len_out": s["kv_len_out"]}


def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    for x in s["planes"]:
        raw = x.view(torch.uint8) if s["case"]["eight"] else x
        raw[:, dst] = raw[:, src]
    return s["planes"]


_PLAIN = {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "keep": _plain_keep, "copy": _plain_copy}


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return _PLAIN[op](s)
    if op == "rotary":
        s["plan"].rotate(s["q"], s["k"], s["q_out"], s["k_out"], positions=s.get("positions"), new_off=s.get("new_off"),
                         kv_len=s.get("kv_len"))
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        s["plan"].append_q8(s["k_new"], s["v_new"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["page_table"],
                            s["new_off"], s["kv_len"], max_new_in_batch=s["sizes"]["max_new_in_batch"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "attend":
        s["plan"].attend_q8(s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["page_table"], s["new_off"],
                            s["kv_len"], s["out"], **s["sizes"])
        return s["out"]
    if op == "keep":
        s["layers"].keep_rows(s["page_table"], s["kv_len"], s["path"], s["acc_len"], s["kv_len_out"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_len_out": s["kv_len_out"]}
    s["layers"].copy_pages(s["src"], s["dst"])
    return s["planes"]


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _round_e4m3(x):
    """x (float64, at most 448 in magnitude) to the nearest e4m3 value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_values(codes, scale, pages, head):
    """Rows of some pages of a head, as the float64 values they stand for."""
    x, p = codes[pages, head].to(torch.float64), scale.view(torch.uint8)[pages, head].to(torch.float64) - 127
    rows, block = x.shape[0] * x.shape[1], x.shape[1] // p.shape[1]
    return (x * torch.exp2(p).repeat_interleave(block, 1)[:, :, None]).reshape(rows, -1)


def _exact_append(case, s, sizes):
    block, page, table, at = case["block"], s["k_pages"].shape[2], s["page_table"].tolist(), 0
    outs = {}
    for name in ("k", "v"):
        codes, power = s[name + "_pages"].to(torch.float64), s[name + "_scale"].view(torch.uint8).to(torch.float64) - 127
        at = 0
        for (n, length), pages in zip(sizes, table):
            for blk in range(length // block, (length + n - 1) // block + 1):
                lo, hi = max(blk * block, length), min((blk + 1) * block, length + n)
                new = s[name + "_new"][at + lo - length:at + hi - length].to(torch.float64).transpose(0, 1)   # [Hkv, rows, D]
                least = torch.ceil(torch.log2(new.abs().amax((1, 2)) / 448)).clamp(min=-126)
                pg, sub, r0 = pages[blk * block // page], blk * block % page // block, blk * block % page
                if lo > blk * block:
                    was = power[pg, :, sub].clone()
                    least = torch.maximum(least, was)
                    rows = slice(r0, r0 + lo - blk * block)
                    codes[pg, :, rows] = _round_e4m3(codes[pg, :, rows] * torch.exp2(was - least)[:, None, None])
                codes[pg, :, r0 + lo - blk * block:r0 + hi - blk * block] = _round_e4m3(new * torch.exp2(-least)[:, None, None])
                power[pg, :, sub] = least
            at += n
        outs[name + "_pages"], outs[name + "_scale"] = codes, torch.exp2(power)
    return outs


def _exact_attend(case, s, sizes):
    h, hkv, d, f64 = case["heads"], case["kv_heads"], case["head_dim"], torch.float64
    table, page, at = s["page_table"].tolist(), s["k_pages"].shape[2], 0
    out = torch.empty(s["q"].shape, dtype=f64, device="cuda")
    for (n, length), pages in zip(sizes, table):
        rows = length + n
        used = pages[:-(-rows // page)]
        for c in range(hkv):
            k = _exact_values(s["k_pages"], s["k_scale"], used, c)[:rows]
            v = _exact_values(s["v_pages"], s["v_scale"], used, c)[:rows]
            for j in range(c * h // hkv, (c + 1) * h // hkv):
                a = s["q"][at:at + n, j].to(f64) @ k.t().contiguous() / math.sqrt(d)
                a.masked_fill_(torch.arange(rows, device="cuda")[None] > length + torch.arange(n, device="cuda")[:, None], -math.inf)
                out[at:at + n, j] = torch.softmax(a, 1) @ v
        at += n
    return out


def exact(case, seed):
    if case["op"] == "rotary":
        s, pos = _rotary_inputs(case, seed)
        r = case["rotary_dim"]
        w = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.tensor(pos, dtype=torch.float64, device="cuda")[:, None] * w)
        outs = {}
        for name in ("q", "k"):
            y = s[name].to(torch.float64).clone()
            shape = y.shape[:2] + ((2, r // 2) if case["layout"] == "half" else (r // 2, 2))
            x = y[..., :r].reshape(shape)
            if case["layout"] == "half":
                x = x.transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(x.contiguous()) * turn[:, None])
            y[..., :r] = (z.transpose(2, 3) if case["layout"] == "half" else z).reshape(y.shape[:2] + (r,))
            outs[name] = y
        return outs
    if case["op"] == "keep":
        s, paths, lens, table = _keep_inputs(case, seed)
        page = s["k_cache"].shape[3]
        for x in (s["k_cache"], s["v_cache"]):
            before = x.clone()
            for p, l, pages in zip(paths, lens, table):
                for i, node in enumerate(p):
                    x[:, pages[(l + i) // page], :, (l + i) % page] = before[:, pages[(l + node) // page], :, (l + node) % page]
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"],
                "kv_len_out": _ints([l + len(p) for l, p in zip(lens, paths)])}
    if case["op"] == "copy":
        s, src, dst = _copy_inputs(case, seed)
        for x in s["planes"]:
            for a, b in zip(src, dst):
                x[:, b].view(torch.uint8).copy_(x[:, a].view(torch.uint8))
        return s["planes"]
    s, sizes = _cache_inputs(case, seed)
    return _exact_append(case, s, sizes) if case["op"] == "append" else _exact_attend(case, s, sizes)
