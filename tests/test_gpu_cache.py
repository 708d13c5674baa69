"""The operators of include/respec_cache.h on the GPU against their definitions in 64 bits (tests/cache_cases.py)."""
import math
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import cache_cases as cc  # noqa: E402
import prompt_cases as pc  # noqa: E402
from test_gpu_prompt import SIZES, _close  # noqa: E402

BF, F32, U8, I32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2511_01282_amd import binding, cache, prompt
    cache.lib()
    return prompt, binding, cache


def _dtype(lib, t):
    return lib[1].BF16 if t == BF else lib[1].F32


def _ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

def _rotary_plan(lib, q, k, r, half, w, amplitude=1.0, **over):
    d = dict(n_q_heads=q.shape[1], n_kv_heads=k.shape[1], head_dim=q.shape[2], rotary_dim=r, dtype=_dtype(lib, q.dtype), frequencies=w,
             layout=lib[2].HALF if half else lib[2].INTERLEAVED, amplitude=amplitude, device="cuda:0")
    return lib[2].RotaryPlan(**dict(d, **over))


def _rows(t, h, hkv, d, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(t, h, d, generator=gen).to(dtype), torch.randn(t, hkv, d, generator=gen).to(dtype)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype,h,hkv,d,r", [
    (BF, 28, 4, 128, 128), (BF, 3, 1, 64, 64), (BF, 8, 8, 128, 32), (BF, 5, 2, 64, 16), (BF, 1, 1, 128, 112), (BF, 70, 70, 64, 48),
    (F32, 4, 4, 64, 64), (F32, 6, 2, 128, 128), (F32, 16, 16, 64, 16), (F32, 33, 1, 128, 80), (F32, 256, 256, 128, 128)])
def test_rotary_at_positions(lib, half, dtype, h, hkv, d, r):
    """One token and many, positions from 0 to the end of 31 bits, far and near ones side by side, tokens left alone."""
    w = lib[2].frequencies(r, 500000.0, scaling="bands", factor=8.0, original_len=8192)
    for t, seed in ((1, 1), (2, 2), (3, 3), (65, 4), (300, 5)):
        if t == 300 and h > 100:
            continue
        q, k = _rows(t, h, hkv, d, dtype, seed)
        rng = random.Random(seed)
        pos = [rng.choice([0, 1, 7, 4095, 131071, 10 ** 6 + 1, (1 << 30) - 1, 2 ** 31 - 1, rng.randrange(1 << 20)]) for _ in range(t)]
        out = [torch.full((t + 1, n, d), 77.0, dtype=dtype, device="cuda") for n in (h, hkv)]
        plan = _rotary_plan(lib, q, k, r, half, w)
        left = [i for i in range(t) if i % 7 == 3]
        given = [-1 - i if i in left else p for i, p in enumerate(pos)]
        plan.rotate(q.cuda(), k.cuda(), out[0][:t], out[1][:t], positions=_ints(given))
        torch.cuda.synchronize()
        for x, y in ((q, out[0].cpu()), (k, out[1].cpu())):
            want, tol = cc.rotary(x, pos, w, r, half)
            for i in left:
                want[i], tol[i] = 77.0, 1e-300
            _close(y[:t], want, tol)
            assert bool((y[t] == 77.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("half", [True, False])
def test_rotary_of_a_batch(lib, dtype, half):
    """Positions of a chunk batch, slices of one projection, in place; an amplitude; rows of no sequence and of bad ones."""
    h, hkv, d, r = 8, 2, 64, 32
    w = lib[2].frequencies(r)
    off, lens = [1, 4, 4, 90, 91, 95, 94], [10, 7, 1000, 2 ** 30 - 1, -5, 0]
    t = 130
    q, k = _rows(t, h, hkv, d, dtype, 6)
    pos = [-1] * t
    for b, l in enumerate(lens[:4]):   # (the fifth's length is negative, the sixth's offsets decrease)
        for i in range(off[b], off[b + 1]):
            pos[i] = l + i - off[b]
    wide = torch.randn(t, h + 2 * hkv, d, device="cuda").to(dtype)
    wide[:, :h], wide[:, h:h + hkv] = q.cuda(), k.cuda()
    before = wide.clone()
    qs, ks = wide[:, :h], wide[:, h:h + hkv]
    st = _ints([-9] * 6)
    plan = _rotary_plan(lib, q, k, r, half, w, amplitude=1.25)
    plan.rotate(qs, ks, qs, ks, new_off=_ints(off), kv_len=_ints(lens), status=st)
    assert st.tolist() == [0, 0, 0, 0, 6, 2]
    for x, y in ((q, qs.cpu()), (k, ks.cpu())):
        want, tol = cc.rotary(x, [max(p, 0) for p in pos], w, r, half, 1.25)
        for i in range(t):
            if pos[i] < 0:
                want[i], tol[i] = x[i].double(), 1e-300
        _close(y, want, tol)
    assert torch.equal(wide[:, h + hkv:], before[:, h + hkv:])
    # one sequence past 2^30 positions; q alone
    st = _ints([-9])
    plan.rotate(qs, None, qs, None, new_off=_ints([0, t]), kv_len=_ints([2 ** 30 - 1]), status=st)
    assert st.tolist() == [6]
    same = qs.clone()
    plan.rotate(qs, None, same, None, positions=_ints([0] * t))
    want, tol = cc.rotary(qs.cpu(), [0] * t, w, r, half, 1.25)
    _close(same.cpu(), want, tol)


def test_rotary_between_rows(lib):
    """Inputs and outputs that lie between each other's rows are no overlap: slices of one array, by heads, by tokens, and with the
    heads ahead of the tokens; sides in place, and one input for all tokens."""
    t, h, hkv, d = 21, 4, 2, 64
    w = lib[2].frequencies(d)
    q, k = _rows(t, h, hkv, d, BF, 10)
    pos = [5 * i for i in range(t)]
    plan = _rotary_plan(lib, q, k, d, True, w)
    want = [cc.rotary(x, pos, w, d, True) for x in (q, k)]
    heads = torch.zeros(t, 2 * (h + hkv) + 1, d, dtype=BF, device="cuda")
    tokens = torch.zeros(2 * t, h + hkv, d, dtype=BF, device="cuda")
    ahead = torch.zeros(2 * (h + hkv), t, d, dtype=BF, device="cuda").transpose(0, 1)
    same = torch.zeros(t, h + hkv, d, dtype=BF, device="cuda")
    for a, b, c, e in ((heads[:, :h], heads[:, h:h + hkv], heads[:, h + hkv:2 * h + hkv], heads[:, 2 * h + hkv:-1]),
                       (tokens[::2, :h], tokens[::2, h:], tokens[1::2, :h], tokens[1::2, h:]),
                       (ahead[:, :2 * h:2], ahead[:, 2 * h::2], ahead[:, 1:2 * h:2], ahead[:, 2 * h + 1::2]),
                       (same[:, :h], same[:, h:], same[:, :h], same[:, h:])):
        a.copy_(q), b.copy_(k)
        plan.rotate(a, b, c, e, positions=_ints(pos))
        _close(c.cpu(), *want[0])
        _close(e.cpu(), *want[1])
    out = torch.zeros(t, h, d, dtype=BF, device="cuda")
    plan.rotate(q[:1].cuda().expand(t, h, d), None, out, None, positions=_ints(pos))
    _close(out.cpu(), *cc.rotary(q[:1].expand(t, h, d), pos, w, d, True))


def test_rotary_of_many_sequences(lib):
    """More sequences than a wave has lanes, most of them empty; more rows than a workgroup takes."""
    rng = random.Random(3)
    counts = [rng.choice([0, 0, 1, 2, 9]) for _ in range(200)]
    lens = [rng.randrange(100000) for _ in counts]
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    for h, hkv, d in ((2, 1, 64), (32, 8, 128)):
        q, k = _rows(off[-1], h, hkv, d, BF, 8)
        w = lib[2].frequencies(d)
        out = torch.empty_like(q, device="cuda"), torch.empty_like(k, device="cuda")
        st = _ints([-9] * 200)
        _rotary_plan(lib, q, k, d, True, w).rotate(q.cuda(), k.cuda(), *out, new_off=_ints(off), kv_len=_ints(lens), status=st)
        assert st.tolist() == [0] * 200
        pos = [l + i for n, l in zip(counts, lens) for i in range(n)]
        for x, y in zip((q, k), out):
            _close(y.cpu(), *cc.rotary(x, pos, w, d, True))


def test_rotary_of_large_calls(lib):
    """As many rows as give a thread several heads, and offsets past 32 bits."""
    h, hkv, d = 28, 4, 128
    q, k = _rows(1500, h, hkv, d, BF, 9)
    w = lib[2].frequencies(d, 1e6)
    for half in (True, False):
        out = torch.empty_like(q, device="cuda"), torch.empty_like(k, device="cuda")
        _rotary_plan(lib, q, k, d, half, w).rotate(q.cuda(), k.cuda(), *out, new_off=_ints([0, 700, 1500]), kv_len=_ints([3, 90000]))
        pos = list(range(3, 703)) + list(range(90000, 90800))
        for x, y in zip((q, k), out):
            _close(y.cpu(), *cc.rotary(x, pos, w, d, half))
    t = 700_000    # 4.6 GB of token rows, queries and keys at their ends
    big = torch.zeros(t, 26, 128, dtype=BF, device="cuda")
    last = torch.randn(2, 1, 128, generator=torch.Generator().manual_seed(1)).to(BF)
    big[-2:, 25:] = last.cuda()
    plan = lib[2].RotaryPlan(n_q_heads=25, n_kv_heads=1, head_dim=128, dtype=lib[1].BF16, frequencies=lib[2].frequencies(128), device="cuda:0")
    plan.rotate(None, big[:, 25:], None, big[:, 25:], new_off=_ints([0, t]), kv_len=_ints([0]))
    _close(big[-2:, 25:].cpu(), *cc.rotary(last, [t - 2, t - 1], lib[2].frequencies(128), 128, True))


def test_rotary_of_nothing(lib):
    plan = lib[2].RotaryPlan(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=lib[1].BF16, device="cuda:0")
    q, k = torch.zeros(3, 4, 64, dtype=BF, device="cuda"), torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    st = _ints([-9, -9])
    plan.rotate(q[:0], k[:0], q[:0], k[:0], new_off=_ints([0, 0, 0]), kv_len=_ints([5, -1]), status=st)
    assert st.tolist() == [0, 6]
    plan.rotate(q[:0], k[:0], q[:0], k[:0], positions=_ints([]))
    plan.rotate(q, k, q, k, new_off=_ints([0]), kv_len=_ints([]))


# ---------------------------------------------------------------------------
# the 8-bit cache
# ---------------------------------------------------------------------------

def _plan(lib, c, **over):
    d = dict(n_q_heads=c.heads, n_kv_heads=c.kv_heads, head_dim=c.head_dim, dtype=_dtype(lib, c.dtype), max_batch=max(len(c.sizes), 1),
             max_new=max(len(c.q), 1), max_kv_len=c.max_kv, device="cuda:0")
    return lib[0].ChunkPlan(**dict(d, **over))


def _cache(x, state, rows_first=False):
    """Codes and scales on the GPU, [page][head][row][D] or as views of [page][row][head][D] and [page][block][head]."""
    def put(t, kind):
        t = t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if rows_first and kind is cc.E4M3 else t.cuda()
        if rows_first and kind is cc.E8M0:   # a stride between heads, and bytes between pages
            wide = torch.full((len(t), t.shape[1], 5, t.shape[2]), 200, dtype=U8, device="cuda")
            wide[:, :, 2] = t
            t = wide[:, :, 2]
        return t.view(kind)
    return (put(state[0], cc.E4M3), put(state[1], cc.E4M3), put(state[2], cc.E8M0), put(state[3], cc.E8M0), x.c.table.cuda(),
            x.c.off.cuda(), x.c.kv_len.cuda())


def _append(lib, x, rows_first=False, fused=False, guard=0):
    c = x.c
    plan = _plan(lib, c, max_new=len(c.q) + guard)
    pad = torch.full((guard, c.kv_heads, c.head_dim), math.nan, dtype=c.dtype)
    k, v = torch.cat([c.k_new, pad]).cuda(), torch.cat([c.v_new, pad]).cuda()
    if fused:
        wide = torch.full((len(k), 3 + 2 * c.kv_heads, c.head_dim), math.nan, dtype=c.dtype, device="cuda")
        wide[:, 3:3 + c.kv_heads], wide[:, 3 + c.kv_heads:] = k, v
        k, v = wide[:, 3:3 + c.kv_heads], wide[:, 3 + c.kv_heads:]
    cache = _cache(x, x.before, rows_first)
    st = _ints([-9] * len(c.sizes))
    plan.append_q8(k, v, *cache, max_new_in_batch=c.max_new, status=st)
    torch.cuda.synchronize()
    assert st.tolist() == [0] * len(c.sizes)
    return [t.view(U8).cpu() for t in cache[:4]]


def _same_state(got, want):
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    assert cc.same_codes(got[0], want[0]) and cc.same_codes(got[1], want[1])


def _attend(lib, x, plan=None, guard=2, rows_first=False, fused=False, scale=None, status=True):
    c = x.c
    plan = plan or _plan(lib, c, max_new=len(c.q) + guard)
    q = torch.cat([c.q, torch.ones(guard, c.heads, c.head_dim, dtype=c.dtype)]).cuda()
    if fused:
        wide = torch.full((len(q), c.heads + 2 * c.kv_heads, c.head_dim), math.nan, dtype=c.dtype, device="cuda")
        wide[:, :c.heads] = q
        q = wide[:, :c.heads]
    out = torch.full((len(q), c.heads, c.head_dim), 77.0, dtype=c.dtype, device="cuda")
    st = _ints([-9] * len(c.sizes)) if status else None
    plan.attend_q8(q, *_cache(x, x.after, rows_first), out, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv, scale=scale, status=st)
    torch.cuda.synchronize()
    if status:
        assert st.tolist() == [0] * len(c.sizes)
    assert bool((out[len(c.q):] == 77.0).all())
    return out[:len(c.q)].cpu()


SHAPES = [(BF, 8, 2, 64, 16, 16), (BF, 4, 4, 128, 48, 16), (BF, 14, 2, 128, 64, 32), (BF, 3, 1, 64, 128, 128), (BF, 16, 1, 128, 64, 64),
          (BF, 5, 5, 64, 1024, 32), (F32, 4, 4, 64, 16, 16), (F32, 6, 2, 128, 96, 32), (F32, 2, 1, 64, 1024, 128)]


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page,block", SHAPES)
def test_append_q8(lib, name, dtype, heads, kv_heads, head_dim, page, block):
    kw = dict(dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block)
    for seed, how in ((1, {}), (2, dict(rows_first=True, fused=True, guard=3))):
        x = cc.q8(SIZES[name], seed=seed, front=(1.0, 0.02)[seed - 1], **kw)
        _same_state(_append(lib, x, **how), x.after)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [16, 64, 128])
def test_append_q8_of_any_values(lib, dtype, block):
    """Zeros, the type's smallest and largest values, NaN and infinities, values on the borders of rounding and of a scale; earlier
    rows whose scale grows and whose small values are rounded again."""
    top = torch.finfo(dtype).max

    def edit(c):
        k, v = c.k_new, c.v_new
        k[0] = 0.0
        k[1, 0], k[1, 1] = 448.0, -449.0
        k[2, 0, :8] = torch.tensor([math.nan, math.inf, -math.inf, 3.0, -3.0, 2.0 ** -130, -2.0 ** -133, 0.0]).to(dtype)
        k[3], k[4] = math.nan, top
        k[5, :, 0], k[5, :, 1] = 2.0 ** -126, 2.0 ** -128
        v[0, :, :16] = 17.0 + torch.arange(16.0).to(dtype)          # ties between two values
        v[0, :, 16] = 448.0
        v[1], v[2] = -math.inf, 1e-30
        v[3:] *= 2.0 ** 40
    for front in (1.0, 1e-4, 0.0, 2.0 ** 60):
        for sizes in ([(6, 3)], [(6, block - 3)], [(6, 0)], [(1, 5), (5, 200)]):
            x = cc.q8(sizes, dtype=dtype, heads=2, kv_heads=2, head_dim=64, page=block * 2, block=block, seed=5, front=front, edit=edit)
            _same_state(_append(lib, x), x.after)


def test_append_q8_token_by_token(lib):
    """A sequence that grows a row at a time and one that is appended whole: the same scales, values off by the roundings that
    larger scales add."""
    c = pc.make([(70, 0)], dtype=F32, heads=2, kv_heads=2, head_dim=64, page=32, seed=3)
    c.k_new *= torch.linspace(0.1, 9.0, 70)[:, None, None]
    x = cc.Q8(c, 16, [torch.zeros(6, 2, 32, 64, dtype=U8)] * 2 + [torch.full((6, 2, 2), 9, dtype=U8)] * 2, None)
    whole, steps = _cache(x, x.before), _cache(x, x.before)
    plan = _plan(lib, c, max_kv_len=100)
    k, v = c.k_new.cuda(), c.v_new.cuda()
    plan.append_q8(k, v, *whole, max_new_in_batch=70)
    for i in range(70):
        plan.append_q8(k[i:i + 1], v[i:i + 1], *steps[:5], _ints([0, 1]), _ints([i]), max_new_in_batch=1)
    assert torch.equal(whole[2].view(U8), steps[2].view(U8)) and torch.equal(whole[3].view(U8), steps[3].view(U8))
    a, b = (torch.stack([cc.values(s[0].view(U8).cpu()[p], s[2].view(U8).cpu()[p].repeat_interleave(16, 1)[..., None]) for p in c.table[0, :3].tolist()])
            for s in (whole, steps))
    # a value of a block with scale 2^k is off by half a step: 2^-4 of itself, or 2^-10 2^k; rounded under a smaller scale before, twice
    byte = torch.stack([whole[2].view(U8).cpu()[p].repeat_interleave(16, 1)[..., None] for p in c.table[0, :3].tolist()])
    tol = a.abs() * 2 ** -4 * 2 + torch.exp2(byte.double() - 127) * 2 ** -10 * 2
    assert bool(((a - b).abs() <= tol).all())


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page,block", SHAPES)
def test_attention_q8(lib, name, dtype, heads, kv_heads, head_dim, page, block):
    x = cc.q8(SIZES[name], dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, seed=len(name))
    _close(_attend(lib, x), *pc.attention(x.c))


@pytest.mark.parametrize("dtype,sizes,kv_heads,group,head_dim,page,block", [
    (BF, [(1, 9000)], 2, 4, 128, 16, 16),
    (BF, [(1, 5000), (1, 20), (1, 2600)], 1, 7, 64, 48, 16),
    (BF, [(33, 4000)], 1, 8, 128, 64, 64),
    (BF, [(300, 1000), (1, 3000), (40, 0)], 2, 1, 64, 96, 32),
    (BF, [(700, 0)], 1, 2, 128, 1024, 128),
    (BF, [(4, 2049), (5, 2047)], 4, 4, 128, 32, 16),
    (BF, [(300, 1000), (1, 3000), (40, 0), (9, 2500)], 2, 4, 128, 16, 16),
    (BF, [(16, 1500), (9, 70), (1, 129)], 2, 4, 64, 16, 16),
    (BF, [(8, 1500), (5, 4000)], 1, 8, 128, 48, 16),
    (BF, [(2, 6000)], 3, 16, 128, 128, 64),
    (BF, [(260, 9000)], 1, 1, 128, 64, 32),
    (F32, [(1, 5000)], 2, 2, 64, 16, 16),
    (F32, [(90, 2000), (1, 100)], 1, 3, 128, 32, 32),
])
def test_attention_q8_long(lib, dtype, sizes, kv_heads, group, head_dim, page, block):
    x = cc.q8(sizes, dtype=dtype, heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, seed=7)
    _close(_attend(lib, x), *pc.attention(x.c))


@pytest.mark.parametrize("sizes", [[(64, 20_000)] + [(64, 7 * i) for i in range(15)], [(1024, 9000)], [(1000, 17_000), (24, 9000)]])
@pytest.mark.parametrize("block", [16, 64])
def test_attention_q8_over_more_tiles_than_a_window(lib, sizes, block):
    """So many rows of queries that the workspace holds no splits, over so many rows that a wave's window of pages and scales moves
    on; a few heads of 256 are checked."""
    h, d, page = 256, 128, 64
    gen = torch.Generator(device="cuda").manual_seed(block)
    pages = [-(-(n + l) // page) for n, l in sizes]
    ids = torch.randperm(sum(pages), generator=gen, device="cuda").tolist()
    shape = (len(ids), h, page, d)
    k, v = (torch.randint(0, 256, shape, dtype=U8, generator=gen, device="cuda") & 0xBF for _ in range(2))   # up to 1.9 in magnitude
    ks, vs = (torch.randint(124, 130, (len(ids), h, page // block), dtype=U8, generator=gen, device="cuda") for _ in range(2))
    table, at = torch.full((len(sizes), max(pages)), -1, dtype=I32), 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor(ids[at:at + n])
        at += n
    total = sum(n for n, _ in sizes)
    q = torch.randn(total, h, d, generator=gen, device="cuda").to(BF)
    off = torch.tensor([0] + [n for n, _ in sizes]).cumsum(0).int()
    lens = torch.tensor([l for _, l in sizes], dtype=I32)
    longest = dict(max_new_in_batch=max(n for n, _ in sizes), max_kv_len_in_batch=max(l for _, l in sizes))
    plan = lib[0].ChunkPlan(n_q_heads=h, n_kv_heads=h, head_dim=d, dtype=lib[1].BF16, max_batch=len(sizes), max_new=total,
                            max_kv_len=longest["max_kv_len_in_batch"], device="cuda:0")
    out = torch.empty_like(q)
    plan.attend_q8(q, k.view(cc.E4M3), v.view(cc.E4M3), ks.view(cc.E8M0), vs.view(cc.E8M0), table.cuda(), off.cuda(), lens.cuda(), out, **longest)
    torch.cuda.synchronize()
    for head in (0, 101, 255):
        rows = []
        for (n, l), t in zip(sizes, table):
            used = t[:-(-(n + l) // page)].long().cuda()
            rows.append(tuple(cc.values(x[used, head].cpu(), s[used, head].cpu().repeat_interleave(block, 1)[..., None]).reshape(-1, 1, d)[:n + l]
                              for x, s in ((k, ks), (v, vs))))
        one = pc.Chunk(BF, 1, 1, d, page, sizes, q[:, head:head + 1].cpu(), None, None, None, None, table, off, lens, rows)
        _close(out[:, head:head + 1].cpu(), *pc.attention(one))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("kind", ["16 rows", "32 rows", "64 rows", "mixed", "long"])
def test_windows_that_move_on_q8(lib, kind, head_dim):
    """Every form of the kernels over so many rows in one split that a wave's window of 64 tiles (of long chunks, 64 units) of
    8192 rows moves on, of few query rows more than once: 256 KV heads and as many tokens as leave the workspace no split, or two at 64 columns,
    whose sequences are as much longer.  A few heads are checked."""
    h, page, block, more = 256, 64, 16, 128 // head_dim
    per = {"16 rows": 16, "32 rows": 32, "64 rows": 64}.get(kind)
    sizes = ([(per, 20_000 * more)] + [(per, 7 * i) for i in range(1024 // per - 1)] if per else
             {"mixed": [(600, 9000 * more), (20, 20_000 * more), (1, 17_500 * more), (403, 100)],
              "long": [(1024, 9000 * more)]}[kind])
    gen = torch.Generator(device="cuda").manual_seed(head_dim)
    pages = [-(-(n + l) // page) for n, l in sizes]
    ids = torch.randperm(sum(pages), generator=gen, device="cuda").tolist()
    k, v = (torch.randint(0, 256, (len(ids), h, page, head_dim), dtype=U8, generator=gen, device="cuda") & 0xBF for _ in range(2))
    ks, vs = (torch.randint(124, 130, (len(ids), h, page // block), dtype=U8, generator=gen, device="cuda") for _ in range(2))
    table, at = torch.full((len(sizes), max(pages)), -1, dtype=I32), 0
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor(ids[at:at + n])
        at += n
    total = sum(n for n, _ in sizes)
    q = torch.randn(total, h, head_dim, generator=gen, device="cuda").to(BF)
    off = torch.tensor([0] + [n for n, _ in sizes]).cumsum(0).int()
    lens = torch.tensor([l for _, l in sizes], dtype=I32)
    longest = dict(max_new_in_batch=max(n for n, _ in sizes), max_kv_len_in_batch=max(l for _, l in sizes))
    plan = lib[0].ChunkPlan(n_q_heads=h, n_kv_heads=h, head_dim=head_dim, dtype=lib[1].BF16, max_batch=len(sizes), max_new=total,
                            max_kv_len=longest["max_kv_len_in_batch"], device="cuda:0")
    out = torch.empty_like(q)
    plan.attend_q8(q, k.view(cc.E4M3), v.view(cc.E4M3), ks.view(cc.E8M0), vs.view(cc.E8M0), table.cuda(), off.cuda(), lens.cuda(), out, **longest)
    torch.cuda.synchronize()
    for head in (0, 255):
        rows = []
        for (n, l), t in zip(sizes, table):
            used = t[:-(-(n + l) // page)].long().cuda()
            rows.append(tuple(cc.values(x[used, head].cpu(), s[used, head].cpu().repeat_interleave(block, 1)[..., None]).reshape(-1, 1, head_dim)[:n + l]
                              for x, s in ((k, ks), (v, vs))))
        one = pc.Chunk(BF, 1, 1, head_dim, page, sizes, q[:, head:head + 1].cpu(), None, None, None, None, table, off, lens, rows)
        _close(out[:, head:head + 1].cpu(), *pc.attention(one))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("step", [32, 128])
def test_numbers_of_splits_q8(lib, head_dim, step):
    for n in (2, 3, 4, 5, 16, 17, 64):
        for more in ([], [(3, 40)]):
            x = cc.q8([(1, n * step - 1)] + more, heads=6, kv_heads=2, head_dim=head_dim, page=32, seed=n)
            _close(_attend(lib, x), *pc.attention(x.c))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_q8_strides_and_scale(lib, dtype):
    x = cc.q8([(3, 100), (20, 30)], dtype=dtype, heads=8, kv_heads=4, head_dim=64, page=32, seed=3)
    _close(_attend(lib, x, rows_first=True, fused=True, scale=0.3, status=False), *pc.attention(x.c, scale=0.3))


def test_attention_q8_in_place(lib):
    x = cc.q8([(1, 3000), (9, 40)], heads=4, kv_heads=2, head_dim=128, page=32, seed=4)
    q = x.c.q.cuda()
    _plan(lib, x.c).attend_q8(q, *_cache(x, x.after), q, max_new_in_batch=x.c.max_new, max_kv_len_in_batch=x.c.max_kv)
    _close(q.cpu(), *pc.attention(x.c))


@pytest.mark.parametrize("dtype,head_dim", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("sizes", [[(40, 25)], [(300, 10)], [(9, 1500)], [(20, 30)], [(1, 9)]])
def test_rows_not_seen_have_no_part_q8(lib, dtype, head_dim, sizes):
    """A new token's NaN or infinite key and value, NaNs in the cache, reach the tokens from it on, and none before; and what lies
    behind the last row (codes and scales of any kind) reaches none."""
    n, l = sizes[0]

    def edit(c):
        for i, (kind, value) in {n - 1: ("v", math.inf), n - 2: ("k", math.nan), n // 2: ("v", -math.inf), n // 2 + 1: ("v", math.nan)}.items():
            if 0 <= i < n and n > 1:
                (c.v_new if kind == "v" else c.k_new)[i, 1, 5 if kind == "v" else 0] = value
    for stale in (cc.NAN_CODE, 0xFF, 0x7E):
        x = cc.q8(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=head_dim, page=32, seed=5, edit=edit, stale=stale)
        _close(_attend(lib, x), *pc.attention(x.c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("byte", [0, 1, 100, 200, 208, 254])
def test_scales_of_any_size(lib, dtype, byte):
    """Values as small as the exponent byte allows, and as large as float32's sums do: a weight is 2^8 at most before the division
    by their sum, so values below 2^(127 - 8) / rows, 2^112 for these 110 rows and 2^89 for 2^30 (448 2^(208 - 127) is under
    2^90), sum up without an infinity.  With byte 254 only zeros do."""
    for sizes in ([(1, 60)], [(70, 40)]):
        x = cc.q8(sizes, dtype=dtype, heads=2, kv_heads=1, head_dim=64, page=16, seed=6)
        c = x.c
        code = [t.clone() for t in x.after[:2]]
        if byte == 254:
            code[1] &= 0x80
        state = [code[0], code[1], torch.ones_like(x.after[2]), torch.full_like(x.after[3], byte)]
        (n, l), rows = sizes[0], c.rows[0]
        out = [torch.empty_like(r) for r in rows]
        for r in range(n + l):
            at, within = int(c.table[0, r // 16]), r % 16
            for which in (0, 1):
                out[which][r] = cc.values(state[which][at, :, within], state[2 + which][at, :, within // 16, None])
        c.rows[0] = tuple(out)
        want, tol = pc.attention(c)
        # below float32's normal numbers (2^-126) a result's step is 2^-133 (bf16) or 2^-149
        tol += (2.0 ** -134 if dtype == BF else 2.0 ** -148) * 2
        x.after = state
        _close(_attend(lib, x), want, tol)


def _with_scales(x, v_bytes):
    """The batch with V's exponent bytes of v_bytes(sequence, row) for every block that holds a row of a sequence."""
    c = x.c
    x.after = [t.clone() for t in x.after]
    for b, (n, l) in enumerate(c.sizes):
        k, v = c.rows[b][0], torch.empty_like(c.rows[b][1])
        for r in range(0, n + l, x.block):
            x.after[3][int(c.table[b, r // c.page]), :, r % c.page // x.block] = v_bytes(b, r)
        for r in range(n + l):
            at, within = int(c.table[b, r // c.page]), r % c.page
            v[r] = cc.values(x.after[1][at, :, within], x.after[3][at, :, within // x.block, None])
        c.rows[b] = (k, v)
    return x


@pytest.mark.parametrize("kind", ["all", "late", "one", "many"])
@pytest.mark.parametrize("dtype,sizes,kv_heads,group,head_dim,page,block", [
    (BF, [(1, 300), (1, 90), (1, 2)], 2, 4, 128, 32, 16),
    (BF, [(1, 3000)], 1, 7, 64, 16, 16),
    (BF, [(4, 2500), (3, 40)], 1, 8, 128, 64, 64),
    (BF, [(8, 0), (8, 100)], 2, 4, 64, 32, 32),
    (BF, [(9, 1500)], 1, 7, 128, 48, 16),
    (BF, [(60, 30), (50, 0)], 2, 1, 64, 16, 16),
    (BF, [(200, 0)], 1, 4, 128, 128, 128),
    (BF, [(150, 2000)], 2, 2, 64, 32, 16),
    (BF, [(90, 2200), (3, 60), (1, 1400), (8, 0)], 1, 4, 128, 16, 16),
    (BF, [(300, 100), (20, 9), (1, 700)], 1, 1, 64, 64, 32),
    (F32, [(1, 900)], 2, 2, 64, 16, 16),
    (F32, [(70, 40), (2, 300)], 1, 3, 128, 32, 32)])
def test_values_as_large_as_the_scales_allow_q8(lib, kind, dtype, sizes, kv_heads, group, head_dim, page, block):
    """Values of up to 448 2^119, whose sums are infinite in float32 and whose means are not: in every block, in those from
    the middle of each sequence on (the tokens before see values of 2^-60, beside them in one group of query rows), in one block,
    and of all kinds."""
    x = cc.q8(sizes, dtype=dtype, heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page=page, block=block, seed=14)
    gen = random.Random(3)
    longest = [n + l for n, l in sizes]
    x = _with_scales(x, {"all": lambda b, r: 246, "late": lambda b, r: 60 if 2 * r < longest[b] else 246,
                         "one": lambda b, r: 245 if r == longest[b] // 3 // block * block else 127,
                         "many": lambda b, r: gen.choice([1, 60, 127, 200, 216, 230, 239, 246])}[kind])
    want, tol = pc.attention(x.c)
    assert float(want.abs().max()) < 2.0 ** 128 * (1 - 2.0 ** -8)
    _close(_attend(lib, x), want, tol)


@pytest.mark.parametrize("dtype,sizes,kv_heads,group,head_dim", [
    (BF, [(1, 300), (1, 40)], 2, 4, 128), (BF, [(8, 100), (3, 20)], 1, 4, 128), (BF, [(9, 60), (8, 90)], 1, 7, 128), (BF, [(3, 100)], 2, 4, 64),
    (BF, [(30, 80)], 2, 2, 64), (BF, [(200, 0)], 1, 4, 128), (BF, [(150, 60), (4, 90)], 2, 2, 64), (F32, [(20, 30)], 1, 2, 64), (BF, [(1, 3000)], 1, 4, 64)])
def test_large_values_in_place_q8(lib, dtype, sizes, kv_heads, group, head_dim):
    """An output in the queries' place, where some columns of some rows have sums that leave float32: what is computed twice has its
    queries twice."""
    x = cc.q8(sizes, dtype=dtype, heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page=32, seed=16)
    x.after = [t.clone() for t in x.after]
    x.after[1][..., 5:] &= 0x80   # (one wave's columns alone are large)
    longest = [n + l for n, l in sizes]
    x = _with_scales(x, lambda b, r: 127 if 2 * r < longest[b] else 246)
    q = x.c.q.cuda()
    _plan(lib, x.c).attend_q8(q, *_cache(x, x.after), q, max_new_in_batch=x.c.max_new, max_kv_len_in_batch=x.c.max_kv)
    _close(q.cpu(), *pc.attention(x.c))


@pytest.mark.parametrize("dtype,head_dim", [(BF, 64), (BF, 128), (F32, 64)])
@pytest.mark.parametrize("sizes", [[(1, 300)], [(200, 40)], [(9, 200), (100, 300)]])
def test_values_behind_float32_q8(lib, dtype, head_dim, sizes):
    """A row with values of 2^128 and more, which float32 does not hold, among ordinary ones: its share of the mean is finite."""
    x = cc.q8(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=head_dim, page=32, seed=15, q_std=0.5)
    x.after = [t.clone() for t in x.after]
    for b, (n, l) in enumerate(sizes):
        r0 = (n + l) // 3 // 16 * 16
        at, within = int(x.c.table[b, r0 // 32]), r0 % 32
        x.after[1][at, :, within:within + 16] &= 0x80
        x.after[1][at, :, within + 3] |= torch.randint(0x70, 0x7E, (2, head_dim), generator=torch.Generator().manual_seed(b), dtype=U8)
    x = _with_scales(x, lambda b, r: 248 if r == sum(sizes[b]) // 3 // 16 * 16 else 127)
    assert max(float(v.abs().max()) for _, v in x.c.rows) >= 2.0 ** 128
    want, tol = pc.attention(x.c)
    assert float(want.abs().max()) < 2.0 ** 128 * (1 - 2.0 ** -8)
    _close(_attend(lib, x), want, tol)


@pytest.mark.parametrize("longest", [0, 70])
def test_many_sequences_q8(lib, longest):
    sizes = [((b * 7) % 4, (b * 13) % 50) for b in range(150)]
    if longest:
        sizes[3], sizes[100] = (longest, 200), (longest - 3, 0)
    x = cc.q8(sizes, heads=2, kv_heads=1, head_dim=64, page=16, seed=2)
    _same_state(_append(lib, x), x.after)
    _close(_attend(lib, x), *pc.attention(x.c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("longest", [5, 90])
def test_bad_sequences_q8(lib, dtype, longest):
    """Bad lengths, offsets and page ids are reported, and the others' rows and blocks are as without them."""
    sizes = [(3, 20), (2, 30), (4, 10), (1, 33), (longest, 17), (2, 2)]
    x = cc.q8(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=64, page=16, seed=8, spare=0)
    c = x.c
    want, tol = pc.attention(c)
    c.kv_len[1], c.kv_len[3] = -1, 10 ** 6
    c.table[2, 0], c.table[4, 1] = 10 ** 6, -7
    c.off[6] = c.off[5] - 1
    st = _ints([0] * 6)
    out = torch.zeros(len(c.q), 4, 64, dtype=dtype, device="cuda")
    plan = _plan(lib, c, max_kv_len=40)
    cache = _cache(x, x.after)
    plan.attend_q8(c.q.cuda(), *cache, out, max_new_in_batch=longest, max_kv_len_in_batch=40, status=st)
    assert st.tolist() == [0, 6, 11, 6, 11, 2]
    _close(out[:3].cpu(), want[:3], tol[:3])
    st.zero_()
    cache = _cache(x, x.before)
    plan.append_q8(c.k_new.cuda(), c.v_new.cuda(), *cache, max_new_in_batch=longest, max_kv_len_in_batch=40, status=st)
    assert st.tolist() == [0, 6, 11, 6, 11, 2]
    mine = c.table[0, :2].tolist()
    others = [p for p in range(len(x.before[0])) if p not in mine + c.table[4].tolist()]
    for got, before, after in zip(cache[:4], x.before, x.after):
        got = got.view(U8).cpu()
        assert cc.same_codes(got[mine], after[mine]) and torch.equal(got[others], before[others])
    plan.attend_q8(c.q.cuda(), *cache, out, max_new_in_batch=2, max_kv_len_in_batch=40, status=st)
    assert st.tolist()[0] == 2


def test_offsets_past_32_bits_q8(lib):
    """A cache of more than 2^32 bytes, read and written behind that."""
    page, d, n_pages = 64, 128, 300_000   # 64 * 128 bytes each, strides of two: 4.9 GB
    k = torch.zeros(n_pages, 2, 1, page, d, dtype=U8, device="cuda")[:, 0]
    v = torch.zeros(n_pages, 2, 1, page, d, dtype=U8, device="cuda")[:, 0]
    ks, vs = (torch.zeros(n_pages, 1, 4, dtype=U8, device="cuda") for _ in range(2))
    assert (n_pages - 1) * k.stride(0) > 2 ** 32
    for sizes in ([(3, 190)], [(70, 123)]):
        x = cc.q8(sizes, heads=4, kv_heads=1, head_dim=d, page=page, seed=9)
        ids = torch.tensor([n_pages - 1, 290_000, 3, n_pages - 2], dtype=I32)
        for j in range(4):
            for t, s in zip((k, v, ks, vs), x.before):
                t[ids[j].item()] = s[x.c.table[0, j]].cuda()
        cache = (k.view(cc.E4M3), v.view(cc.E4M3), ks.view(cc.E8M0), vs.view(cc.E8M0), ids[None].cuda(), x.c.off.cuda(), x.c.kv_len.cuda())
        plan = _plan(lib, x.c)
        plan.append_q8(x.c.k_new.cuda(), x.c.v_new.cuda(), *cache, max_new_in_batch=x.c.max_new)
        out = torch.empty(len(x.c.q), 4, d, dtype=BF, device="cuda")
        plan.attend_q8(x.c.q.cuda(), *cache, out, max_new_in_batch=x.c.max_new, max_kv_len_in_batch=x.c.max_kv)
        _close(out.cpu(), *pc.attention(x.c))


def test_nothing_to_do_q8(lib):
    for sizes in ([], [(0, 5), (0, 0)]):
        x = cc.q8(sizes, heads=4, kv_heads=2, head_dim=64, page=16)
        plan = _plan(lib, x.c, max_batch=2, max_new=4, max_kv_len=10)
        st = _ints([-9] * len(sizes))
        out = torch.full((4, 4, 64), 7.0, dtype=BF, device="cuda")
        cache = _cache(x, x.before)
        plan.attend_q8(out[:0], *cache, out[:0], max_new_in_batch=0, max_kv_len_in_batch=10, status=st)
        assert st.tolist() == [0] * len(sizes)
        st.fill_(-9)
        plan.append_q8(x.c.k_new.cuda(), x.c.v_new.cuda(), *cache, max_new_in_batch=0, status=st)
        assert st.tolist() == [0] * len(sizes) and bool((out == 7.0).all())
        assert all(torch.equal(t.view(U8).cpu(), b) for t, b in zip(cache, x.before))


def test_two_plans_at_once_q8(lib):
    """Calls that overlap on two streams, a workspace each; the results repeat bit for bit."""
    runs = []
    for d in (64, 128):
        x = cc.q8([(1, 4000), (70, 600)], heads=8, kv_heads=2, head_dim=d, page=16, seed=20 + d)
        q = x.c.q.cuda()
        runs.append((_plan(lib, x.c), q, _cache(x, x.after), torch.empty_like(q), torch.empty_like(q), torch.cuda.Stream(), x.c))
    for plan, q, cache, out, first, stream, c in runs:
        plan.attend_q8(q, *cache, first, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv)
    torch.cuda.synchronize()
    for _ in range(20):
        for plan, q, cache, out, first, stream, c in runs:
            plan.attend_q8(q, *cache, out, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv, stream=stream)
    torch.cuda.synchronize()
    for plan, q, cache, out, first, stream, c in runs:
        assert torch.equal(out, first)
        _close(out.cpu(), *pc.attention(c))


def _chain(lib, x, plan, rotary, qk, cache, turned, out):
    """New tokens turned to their positions, appended and attended to, as a decoding step does."""
    off, lens = cache[5], cache[6]
    rotary.rotate(qk[0], qk[1], turned[0], turned[1], new_off=off, kv_len=lens)
    plan.append_q8(turned[1], qk[2], *cache, max_new_in_batch=x.c.max_new)
    plan.attend_q8(turned[0], *cache, out, max_new_in_batch=x.c.max_new, max_kv_len_in_batch=x.c.max_kv)


def test_captured_decoding_step_replays(lib):
    """Rotary positions, append and attention captured once, replayed with other lengths and tokens, eager work in between; every
    replay against the eager calls, bit for bit."""
    x = cc.q8([(5, 150), (1, 300), (0, 7), (3, 64)], heads=4, kv_heads=2, head_dim=64, page=16, seed=12, spare=20)
    c = x.c
    used = set(c.table[c.table >= 0].tolist())
    c.table[c.table < 0] = [p for p in range(len(c.k_pages)) if p not in used][0]
    gen = torch.Generator(device="cuda").manual_seed(3)
    qk = [t.cuda() for t in (c.q, c.k_new, c.v_new)]
    rotary = lib[2].RotaryPlan(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=lib[1].BF16, device="cuda:0")

    def buffers():
        return _cache(x, x.before), [torch.zeros_like(t) for t in qk[:2]], torch.zeros_like(qk[0]), _plan(lib, c, max_kv_len=300)

    cache, turned, out, plan = buffers()
    e_cache, e_turned, e_out, e_plan = buffers()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _chain(lib, x, plan, rotary, qk, cache, turned, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(lib, x, plan, rotary, qk, cache, turned, out)
    for k, (off, lens) in enumerate([([0, 5, 6, 6, 9], [150, 300, 7, 64]), ([0, 1, 2, 4, 5], [3, 299, 0, 80]),
                                     ([0, 5, 6, 6, 9], [150, 300, 7, 64]), ([2, 2, 3, 3, 9], [10, 160, 7, 5])]):
        for t, v in ((cache[5], off), (cache[6], lens)):
            t.copy_(torch.tensor(v, dtype=I32))
        for t in qk:
            t.normal_(generator=gen)
        for a, b in zip(e_cache[:4] + e_cache[5:], cache[:4] + cache[5:]):
            a.view(U8).copy_(b.view(U8))
        e_out.copy_(out)
        graph.replay()
        torch.cuda.synchronize()
        _chain(lib, x, e_plan, rotary, qk, e_cache, e_turned, e_out)
        torch.cuda.synchronize()
        assert torch.equal(out[off[0]:off[-1]].view(U8), e_out[off[0]:off[-1]].view(U8)), k   # (NaN where stale rows are seen)
        assert all(torch.equal(a.view(U8), b.view(U8)) for a, b in zip(cache[:4], e_cache[:4])), k


def test_captured_sequences_that_grow(lib):
    """A step captured once whose lengths grow by its tokens, on the device, replayed until every sequence has gone into new blocks
    and pages; every replay against the eager calls, bit for bit, and the last one against the definition over the cache's values."""
    news, start, page, longest = [3, 1, 0, 6], [10, 31, 7, 0], 16, 120
    c = pc.make([(n, longest - n) for n in news], heads=4, kv_heads=2, head_dim=64, page=page, seed=13)
    x = cc.Q8(c, 16, [torch.full((len(c.k_pages), 2, page, 64), cc.NAN_CODE, dtype=U8)] * 2 + [torch.zeros(len(c.k_pages), 2, 1, dtype=U8)] * 2, None)
    rotary = lib[2].RotaryPlan(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=lib[1].BF16, device="cuda:0")
    gen = torch.Generator(device="cuda").manual_seed(4)
    qk, counts = [t.cuda() for t in (c.q, c.k_new, c.v_new)], _ints(news)

    def side():
        cache, plan = _cache(x, x.before), _plan(lib, c, max_kv_len=longest)
        for t in cache[:2]:   # (rows in front: a value of every row)
            t.view(U8).fill_(0x38)
        cache[2].view(U8).fill_(120), cache[3].view(U8).fill_(125)
        cache[6].copy_(torch.tensor(start, dtype=I32))
        turned, out = [torch.zeros_like(t) for t in qk[:2]], torch.zeros_like(qk[0])

        def step():
            rotary.rotate(qk[0], qk[1], turned[0], turned[1], new_off=cache[5], kv_len=cache[6])
            plan.append_q8(turned[1], qk[2], *cache, max_new_in_batch=6)
            plan.attend_q8(turned[0], *cache, out, max_new_in_batch=6, max_kv_len_in_batch=longest)
            cache[6].add_(counts)
        return cache, turned, out, step

    cache, turned, out, step = side()
    e_cache, e_turned, e_out, e_step = side()
    apart = torch.cuda.Stream()
    with torch.cuda.stream(apart):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for a, b in zip(cache, e_cache):
        a.view(U8).copy_(b.view(U8))
    for k in range(17):
        for t in qk:
            t.normal_(generator=gen)
        lens = cache[6].tolist()
        graph.replay()
        torch.cuda.synchronize()
        e_step()
        torch.cuda.synchronize()
        assert torch.equal(out, e_out) and all(torch.equal(a.view(U8), b.view(U8)) for a, b in zip(cache, e_cache)), k
        if k % 4 == 0:
            state = [t.view(U8).cpu() for t in cache[:4]]
            c.sizes, c.q, c.rows = [(n, l) for n, l in zip(news, lens)], turned[0].cpu(), []
            for (n, l), pages in zip(c.sizes, c.table.tolist()):
                at = [(pages[r // page], r % page) for r in range(n + l)]
                c.rows.append(tuple(torch.stack([cc.values(state[w][p, :, i], state[2 + w][p, :, 0, None]) for p, i in at]) if at else None
                                    for w in (0, 1)))
            _close(out.cpu(), *pc.attention(c))
    assert cache[6].tolist() == [l + 17 * n for l, n in zip(start, news)]


# ---------------------------------------------------------------------------
# rows kept
# ---------------------------------------------------------------------------

def _keep_case(rng, batch, layers, heads, d, page, dtype, nodes=26, layout="paged"):
    lens = [rng.choice([0, 1, 15, 16, 100, rng.randrange(300)]) for _ in range(batch)]
    acc = [min(nodes - 1, rng.choice([-1, 0, 1, 3, 12, rng.randrange(nodes)])) for _ in range(batch)]
    pages = [-(-(l + nodes) // page) for l in lens]
    ids = list(range(sum(pages) + 2))
    rng.shuffle(ids)
    table, at = [], 0
    for n in pages:
        table.append(ids[at:at + n] + [-1] * (max(pages) - n))
        at += n
    paths = [[0] + sorted(rng.sample(range(1, nodes), a)) if a >= 0 else [] for a in acc]
    shape = (layers, len(ids), heads, page, d) if layout == "paged" else (layers, len(ids), page, heads, d)
    gen = torch.Generator().manual_seed(rng.randrange(1 << 30))
    k, v = (torch.randn(shape, generator=gen).to(dtype) for _ in range(2))
    if layout != "paged":
        k, v = k.transpose(2, 3), v.transpose(2, 3)
    return lens, acc, paths, table, k, v


def _kept(t, lens, paths, table, page):
    """The definition, on a copy."""
    want = t.clone()
    for l, p, pages in zip(lens, paths, table):
        for i, node in enumerate(p):
            want[:, pages[(l + i) // page], :, (l + i) % page] = t[:, pages[(l + node) // page], :, (l + node) % page]
    return want


@pytest.mark.parametrize("dtype,heads,d,page,layers,layout", [
    (BF, 8, 128, 16, 3, "paged"), (BF, 1, 64, 7, 1, "paged"), (BF, 4, 128, 400, 2, "rows"), (F32, 3, 64, 24, 5, "rows"),
    (F32, 2, 128, 64, 1, "paged"), (BF, 33, 64, 1, 2, "paged")])
@pytest.mark.parametrize("nodes", [1, 2, 26, 65])
def test_keep_rows(lib, dtype, heads, d, page, layers, layout, nodes):
    """Paths that overlap the rows that they move to, failed sequences (-1), roots alone, whole trees."""
    rng = random.Random(nodes)
    for batch in (1, 6):
        lens, acc, paths, table, k, v = _keep_case(rng, batch, layers, heads, d, page, dtype, nodes, layout)
        kg, vg = k.cuda(), v.cuda()
        out, st = _ints([-9] * batch), _ints([-9] * batch)
        path = _ints([p + [-1] * (nodes + 1 - len(p)) for p in paths])[:, :nodes]   # (rows further apart than their width)
        lib[2].CacheLayers(kg, vg).keep_rows(_ints(table), _ints(lens), path, _ints(acc), out, status=st)
        assert st.tolist() == [0] * batch and out.tolist() == [l + len(p) for l, p in zip(lens, paths)]
        assert torch.equal(kg.cpu(), _kept(k, lens, paths, table, page)) and torch.equal(vg.cpu(), _kept(v, lens, paths, table, page))


def test_keep_rows_refuses_bad_sequences(lib):
    """Each is reported and left as it was; the others are moved."""
    page, nodes = 16, 10
    good = [0, 3, 5, 9, -1, -1, -1]
    paths = [good, [0, 3, 3] + [-1] * 4, [0, 5, 4] + [-1] * 4, [-1, 2, 3] + [-1] * 4, good, good, good, good, good, good]
    acc = [3, 2, 2, 2, -2, 7, 3, 3, 3, 3]
    lens = [20, 20, 20, 20, 20, 20, -1, 23, 20, 2 ** 31 - 1]
    want = [0, 5, 5, 5, 5, 5, 6, 6, 11, 6]
    table = [[2 * b, 2 * b + 1] for b in range(10)]
    table[8] = [16, 99]
    gen = torch.Generator().manual_seed(1)
    k = torch.randn(2, 20, 2, page, 64, generator=gen).to(BF)
    kg, vg = k.cuda(), k.cuda()
    out, st = _ints([-9] * 10), _ints([-9] * 10)
    lib[2].CacheLayers(kg, vg).keep_rows(_ints(table), _ints(lens), _ints(paths), _ints(acc), out, status=st)
    assert st.tolist() == want and out.tolist() == [24] + lens[1:]
    expected = _kept(k, lens[:1], [good[:4]], table[:1], page)
    assert torch.equal(kg.cpu(), expected) and torch.equal(vg.cpu(), expected)
    # the last row that the pages hold, and one more
    for l, status in ((22, 0), (23, 6)):
        st.fill_(-9)
        lib[2].CacheLayers(kg, vg).keep_rows(_ints(table[:1]), _ints([l]), _ints([good]), _ints([3]), status=st[:1])
        assert st.tolist()[0] == status


def test_keep_rows_past_32_bits(lib):
    """Layers more than 2^32 bytes apart."""
    k = torch.zeros(2, 17_000, 8, 64, 128, dtype=BF, device="cuda")   # 2.2 GB a layer
    v = torch.zeros(2, 17_000, 8, 64, 128, dtype=BF, device="cuda")
    assert k.stride(0) * 2 * 2 > 2 ** 32
    k[1, 16_999, :, 5], v[1, 16_999, :, 5] = 3.0, 4.0
    lib[2].CacheLayers(k, v).keep_rows(_ints([[16_999]]), _ints([1]), _ints([[0, 4]]), _ints([1]))
    assert bool((k[1, 16_999, :, 2] == 3.0).all()) and bool((v[1, 16_999, :, 2] == 4.0).all())
    assert int((k != 0).sum()) == 2 * 8 * 128


def test_keep_writes_in_gaps_of_what_it_reads(lib):
    """New lengths and statuses in the gaps between the paths' rows and the page table's, as columns of one array of integers."""
    rng = random.Random(5)
    lens, acc, paths, table, k, v = _keep_case(rng, 3, 2, 2, 64, 16, BF)
    wide = _ints([p + [-1] * (26 - len(p)) + [-9] * 3 for p in paths])
    pages = _ints([t + [-9] * 3 for t in table])
    path, out, st = wide[:, :26], wide[1, 26:], pages[0, len(table[0]):]
    kg, vg = k.cuda(), v.cuda()
    lib[2].CacheLayers(kg, vg).keep_rows(pages[:, :len(table[0])], _ints(lens), path, _ints(acc), out, status=st)
    assert st.tolist() == [0] * 3 and out.tolist() == [l + len(p) for l, p in zip(lens, paths)]
    assert torch.equal(kg.cpu(), _kept(k, lens, paths, table, 16)) and torch.equal(vg.cpu(), _kept(v, lens, paths, table, 16))
    assert bool((wide[0, 26:] == -9).all()) and bool((wide[2, 26:] == -9).all()) and bool((pages[1:, len(table[0]):] == -9).all())


def test_captured_keep_replays(lib):
    """Captured once, replayed on other caches' contents, lengths and paths (failed sequences among them), eager work in between."""
    rng = random.Random(11)
    nodes, page, batch = 20, 16, 5
    shape = (3, 40, 2, page, 64)
    k, v = (torch.zeros(shape, dtype=BF, device="cuda") for _ in range(2))
    table = torch.arange(40, dtype=I32, device="cuda").view(batch, 8)
    lens, path, acc, out, st = _ints([0] * batch), _ints([[0] * nodes] * batch), _ints([0] * batch), _ints([0] * batch), _ints([0] * batch)
    layers = lib[2].CacheLayers(k, v)
    layers.keep_rows(table, lens, path, acc, out, status=st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layers.keep_rows(table, lens, path, acc, out, status=st)
    for _ in range(4):
        accs = [rng.choice([-1, 0, 5, nodes - 1, nodes]) for _ in range(batch)]   # (the last: one more than the path holds)
        paths = [[0] + sorted(rng.sample(range(1, nodes), min(max(a, 0), nodes - 1))) for a in accs]
        ls = [rng.randrange(8 * page - nodes) for _ in range(batch)]
        for t, x in ((lens, ls), (acc, accs), (path, [p + [-1] * (nodes - len(p)) for p in paths])):
            t.copy_(torch.tensor(x, dtype=I32))
        kc, vc = k.normal_().cpu(), v.normal_().cpu()
        graph.replay()
        torch.cuda.synchronize()
        kept = [p if 0 <= a < nodes else [] for p, a in zip(paths, accs)]
        assert st.tolist() == [5 if a == nodes else 0 for a in accs] and out.tolist() == [l + len(p) for l, p in zip(ls, kept)]
        assert torch.equal(k.cpu(), _kept(kc, ls, kept, table.tolist(), page)) and torch.equal(v.cpu(), _kept(vc, ls, kept, table.tolist(), page))


def test_verification_then_kept_rows(lib):
    """Verification steps whose accepted rows are kept in the cache, and nothing else of their trees: the next step's attention is
    that over a cache of the accepted tokens alone."""
    import numpy as np
    import decode_loop
    from paper_2511_01282_amd import runner
    m = decode_loop.make_model(n_heads=4, head_dim=64, hidden=256)
    s = m.shape
    text = [int(t) for t in decode_loop.prompt()[:20]]
    cap = 64
    w = decode_loop.workload(m, text, [-1], [text[-1]], [0])
    ref = runner.run(w, device="cuda:0")
    first = int(ref["argmax"][0])
    # a tree whose right continuation is not its first branch: the root, two wrong nodes, the model's own tokens behind them
    tokens, parents = [text[-1], (first + 1) % s.vocab, (first + 2) % s.vocab, first], [-1, 0, 0, 0]
    nxt = int(runner.run(decode_loop.workload(m, text + [first], [-1], [first], [0]), device="cuda:0")["argmax"][0])
    tokens, parents = tokens + [(nxt + 1) % s.vocab, nxt], parents + [3, 3]
    w = decode_loop.workload(m, text, parents, tokens, [0] * 6)
    ins, kw = runner.upload(w, "cuda:0"), runner.step_kwargs(w)
    L, d = int(w.kv_len[0]), s.head_dim
    k, v = (torch.zeros(1, s.n_kv_heads, cap, d, device="cuda") for _ in range(2))
    k[:, :, :w.k_cache.shape[2]], v[:, :, :w.k_cache.shape[2]] = ins["k_cache"], ins["v_cache"]
    ins["k_cache"], ins["v_cache"], kw["kv_capacity"] = k, v, cap
    plan = runner.make_plan(w, "cuda:0")
    from paper_2511_01282_amd import binding
    out = binding.alloc_outputs(total_nodes=6, batch=1, hidden=s.hidden, vocab=s.vocab, topk_out=s.topk_out, max_depth=s.max_depth, device="cuda:0")
    plan.step(ins, out, **kw)
    new_len, table = _ints([0]), _ints([[0]])
    lib[2].CacheLayers(k, v).keep_rows(table, ins["kv_len"], out["path"], out["acc_len"], new_len)
    assert out["path"][0, :3].tolist() == [0, 3, 5] and new_len.tolist() == [L + 3]
    accepted = text + [first, nxt]
    want = decode_loop.workload(m, accepted, [-1], [accepted[-1]], [0])
    rows = L + 3
    torch.testing.assert_close(k[:, :, :rows].cpu(), torch.from_numpy(np.ascontiguousarray(want.k_cache[:, :, :rows])), rtol=0, atol=0)
    torch.testing.assert_close(v[:, :, :rows].cpu(), torch.from_numpy(np.ascontiguousarray(want.v_cache[:, :, :rows])), rtol=0, atol=0)


def test_steps_over_kept_rows(lib):
    """Verification steps of two sequences over one cache: each step's accepted rows are kept, and the next step reads them with the
    lengths that the call before left on the device.  Every output is that of a step over caches built afresh, bit for bit; a second
    layer's rows move along."""
    import decode_loop
    from paper_2511_01282_amd import binding, runner
    m = decode_loop.make_model(n_heads=4, head_dim=64, hidden=256)
    s, cap = m.shape, 96
    prompt = [int(t) for t in decode_loop.prompt()]
    texts, heads, d = [prompt[:20], prompt[3:44]], s.n_kv_heads, s.head_dim
    tables = [torch.from_numpy(t).view(-1, heads, d) for t in (m.E_k, m.E_v)]
    caches = [torch.full((2, 2, heads, cap, d), math.nan, device="cuda") for _ in tables]

    def put(to, table, b, first, tokens, factor=1.0):
        to[b, :, first:first + len(tokens)] = table[tokens].transpose(0, 1).to(to.device) * factor

    for b, text in enumerate(texts):
        for t, table in zip(caches, tables):
            put(t[0], table, b, 0, text[:-1])
            put(t[1], table, b, 0, text[:-1], 2.0)
    lens, pages, layers = _ints([len(t) - 1 for t in texts]), _ints([[0], [1]]), lib[2].CacheLayers(*caches)
    accepted = set()
    for step in range(5):
        trees = []
        for b, text in enumerate(texts):
            right, at = [], list(text)
            for _ in range(3):
                right.append(int(runner.run(decode_loop.workload(m, at, [-1], [at[-1]], [0]), device="cuda:0")["argmax"][0]))
                at.append(right[-1])
            wrong = [(t + 1) % s.vocab for t in right]
            if (step + b) % 3 == 2:   # no node but the root is right
                trees.append(([text[-1], wrong[0]], [-1, 0]))
            else:                     # two or three are, behind wrong ones
                n = 6 + 2 * (step % 2)
                trees.append(([text[-1], wrong[0], wrong[1], right[0], wrong[1], right[1], wrong[2], right[2]][:n], [-1, 0, 1, 0, 3, 3, 5, 5][:n]))
        loads = [decode_loop.workload(m, text, parents, tokens, [0] * len(tokens)) for text, (tokens, parents) in zip(texts, trees)]
        ins = [runner.upload(w, "cuda:0") for w in loads]
        both = {n: torch.cat([i[n] for i in ins]) for n in ("hidden", "parent", "token", "src")}
        sizes = [len(t) for t, _ in trees]
        both.update(lm_head=ins[0]["lm_head"], node_off=_ints([0, sizes[0], sum(sizes)]))
        fresh = [torch.zeros(2, heads, cap, d, device="cuda") for _ in tables]
        for b, (text, (tokens, _)) in enumerate(zip(texts, trees)):
            for t, f, table in zip(caches, fresh, tables):
                put(f, table, b, 0, text[:-1] + tokens)
                put(t[0], table, b, len(text) - 1, tokens)
                put(t[1], table, b, len(text) - 1, tokens, 2.0)
        kw = dict(runner.step_kwargs(loads[0]), batch=2, total_nodes=sum(sizes), max_nodes_in_batch=max(sizes),
                  max_kv_len_in_batch=max(len(t) - 1 for t in texts), kv_capacity=cap)
        plan = runner.make_plan(loads[0], "cuda:0", max_batch=2, max_nodes=8, max_kv_len=cap)
        outs = []
        for (k, v), length in (((caches[0][0], caches[1][0]), lens), (fresh, _ints([len(t) - 1 for t in texts]))):
            out = binding.alloc_outputs(total_nodes=sum(sizes), batch=2, hidden=s.hidden, vocab=s.vocab, topk_out=s.topk_out, max_depth=s.max_depth,
                                        device="cuda:0", attn_out=True)
            for t in out.values():   # (a strict step leaves some outputs alone)
                if t is not None:
                    t.zero_()
            plan.step(dict(both, k_cache=k, v_cache=v, kv_len=length), out, **kw)
            outs.append(out)
        for name, t in outs[0].items():
            assert t is None or torch.equal(t, outs[1][name]), (step, name)
        new, st = _ints([-1, -1]), _ints([-1, -1])
        layers.keep_rows(pages, lens, outs[0]["path"], outs[0]["acc_len"], new, status=st)
        for b, (tokens, _) in enumerate(trees):
            acc = int(outs[0]["acc_len"][b])
            path = outs[0]["path"][b, :acc + 1].tolist()
            accepted.add(acc)
            texts[b] = texts[b] + [tokens[i] for i in path[1:]] + [int(outs[0]["bonus"][b])]
            for t, table in zip(caches, tables):
                rows = table[texts[b][:-1]].transpose(0, 1)
                assert torch.equal(t[0, b, :, :rows.shape[1]].cpu(), rows) and torch.equal(t[1, b, :, :rows.shape[1]].cpu(), rows * 2)
        assert st.tolist() == [0, 0] and new.tolist() == [len(t) - 1 for t in texts]
        lens = new
    assert accepted >= {0, 2, 3}


# ---------------------------------------------------------------------------
# pages copied
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("layers,pages,heads,page,d,block", [(1, 5, 1, 16, 64, 16), (3, 9, 5, 48, 128, 16), (2, 40, 8, 128, 64, 32),
                                                             (4, 6, 3, 1, 128, 1), (2, 7, 2, 37, 40, 37), (1, 12, 3, 9, 5, 3)])
def test_copy_pages(lib, eight, layers, pages, heads, page, d, block):
    rng = random.Random(pages)
    gen = torch.Generator().manual_seed(pages)
    k, v = (torch.randint(0, 256, (layers, pages, heads, page, d * (1 if eight else 2)), generator=gen, dtype=U8) for _ in range(2))
    t = [k.view(cc.E4M3), v.view(cc.E4M3)] if eight else [k.view(BF), v.view(BF)]
    if eight:
        t += [torch.randint(0, 256, (layers, pages, heads, page // block), generator=gen, dtype=U8).view(cc.E8M0) for _ in range(2)]
    n = max(1, pages // 3)
    ids = list(range(pages))
    rng.shuffle(ids)
    src, dst = [ids[n + rng.randrange(pages - n)] for _ in range(n)] + [-1, pages, 0, -2], ids[:n] + [ids[0], ids[0], pages, ids[0]]
    src, dst = src + [ids[-1]], dst + [ids[-1]]
    for rows_first in (False, True):
        g = [x.cuda() for x in t]
        if rows_first:   # views of [layer][row][page][head]..., and of rows further apart
            g = [torch.nn.functional.pad(x.view(U8), (0, x.element_size() * 3)).permute(0, 3, 1, 2, 4).contiguous().permute(0, 2, 3, 1, 4)[..., :-3 * x.element_size()]
                 if x.dim() == 5 else x.view(U8).transpose(1, 2).contiguous().transpose(1, 2) for x in g]
            if not eight and g[0].stride(3) % 2 == 0 and g[0].stride(2) % 2 == 0:
                g = [x.view(BF) for x in g]
            elif eight:
                g = [x.view(cc.E4M3) if x.dim() == 5 else x.view(cc.E8M0) for x in g]
            else:
                continue
        before = [x.view(U8).clone() if not rows_first else x.clone() for x in g]
        st = _ints([-9] * len(src))
        lib[2].CacheLayers(*g).copy_pages(_ints(src), _ints(dst), status=st)
        assert st.tolist() == [0] * n + [0, 11, 11, 11, 0]
        for x, b in zip(g, before):
            want = b.clone()
            raw, was = want.view(U8), b.view(U8)
            for i, j in zip(src[:n], dst[:n]):
                raw[:, j] = was[:, i]
            assert torch.equal(x.view(U8), want.view(U8))


def test_copy_pages_of_one_layer_and_none(lib):
    k = torch.randn(6, 2, 16, 64, device="cuda")
    v, before = k + 1, k.clone()
    layers = lib[2].CacheLayers(k, v)
    layers.copy_pages(_ints([]), _ints([]))
    layers.copy_pages(_ints([-1, -1]), _ints([2, 3]))
    assert torch.equal(k, before)
    layers.copy_pages(_ints([4]), _ints([1]))
    assert torch.equal(k[1], before[4]) and torch.equal(v[1], before[4] + 1) and torch.equal(k[2:], before[2:])


def test_fork_then_append(lib):
    """Two samples go on from one prompt: its whole pages are shared, its partly filled one is copied, both append rows of their own
    and attend; and the steps repeat from a captured graph."""
    n, l, page = 3, 37, 16
    x = cc.q8([(n, l), (n, l)], heads=4, kv_heads=2, head_dim=64, page=page, block=16, seed=31)
    c = x.c
    one = c.table[0].clone()
    c.table[1, :2] = one[:2]                       # rows 0 - 31
    fresh = int(c.table[1, 2])
    c.rows[1] = tuple(torch.empty_like(r) for r in c.rows[0])
    code = [x.before[0].clone(), x.before[1].clone(), x.before[2].clone(), x.before[3].clone()]
    for t in code:
        t[fresh] = t[int(one[2])]
    done = n
    for which in (0, 1):
        cc.append(code[which], code[2 + which], (c.k_new, c.v_new)[which][done:done + n].double(), c.table[1], l, page, 16)
        for r in range(n + l):
            at, within = int(c.table[1, r // page]), r % page
            c.rows[1][which][r] = cc.values(code[which][at, :, within], code[2 + which][at, :, within // 16, None])
    want, tol = pc.attention(c)
    cache = _cache(x, x.before)
    layers = lib[2].CacheLayers(*cache[:4])
    plan = _plan(lib, c)
    src, dst = _ints([int(one[2])]), _ints([fresh])
    rows, q, out = [c.k_new.cuda(), c.v_new.cuda()], c.q.cuda(), torch.empty_like(c.q, device="cuda")

    def step():
        layers.copy_pages(src, dst)
        plan.append_q8(*rows, *cache, max_new_in_batch=n)
        plan.attend_q8(q, *cache, out, max_new_in_batch=n, max_kv_len_in_batch=l)

    start = [t.view(U8).clone() for t in cache[:4]]
    step()
    _close(out.cpu(), want, tol)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t, s in zip(cache[:4], start):
            t.view(U8).copy_(s)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _close(out.cpu(), want, tol)


@pytest.mark.parametrize("op", ["rotary", "append", "keep", "copy"])
def test_calls_on_another_stream(lib, op):
    """A call on a stream that the caller names waits for what is before it there."""
    side = torch.cuda.Stream()
    x = cc.q8([(4, 30)], heads=4, kv_heads=2, head_dim=64, page=16, seed=40)
    c, cache = x.c, None
    cache = _cache(x, x.before)
    k = torch.randn(2, 6, 2, 16, 64, device="cuda").to(BF)
    want = k.clone()
    q, kn, vn = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda()
    q_late, kn_late, k_late = torch.zeros_like(q), torch.zeros_like(kn), torch.zeros_like(k)
    out = torch.zeros_like(q), torch.zeros_like(kn)
    table, lens, path, acc, src, dst, pos = _ints([[0, 1]]), _ints([3]), _ints([[0, 2]]), _ints([1]), _ints([1]), _ints([4]), _ints([5, 6, 7, 8])
    w = lib[2].frequencies(64)
    rotary, plan, layers = _rotary_plan(lib, c.q, c.k_new, 64, True, w), _plan(lib, c), lib[2].CacheLayers(k_late, k_late.clone())
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        q_late.copy_(q), kn_late.copy_(kn), k_late.copy_(k)
    if op == "rotary":
        rotary.rotate(q_late, kn_late, *out, positions=pos, stream=side)
        side.synchronize()
        _close(out[0].cpu(), *cc.rotary(c.q, [5, 6, 7, 8], w, 64, True))
    elif op == "append":
        plan.append_q8(kn_late, vn, *cache, max_new_in_batch=4, stream=side)
        side.synchronize()
        _same_state([t.view(U8).cpu() for t in cache[:4]], x.after)
    elif op == "keep":
        layers.keep_rows(table, lens, path, acc, stream=side)
        side.synchronize()
        want[:, 0, :, 4] = k[:, 0, :, 5]
        assert torch.equal(k_late, want)
    else:
        layers.copy_pages(src, dst, stream=side)
        side.synchronize()
        want[:, 4] = k[:, 1]
        assert torch.equal(k_late, want)
    torch.cuda.synchronize()
