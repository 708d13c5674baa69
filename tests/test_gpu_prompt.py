"""The prompt side on the GPU against the operators in 64 bits (tests/prompt_cases.py)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import prompt_cases as pc  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2511_01282_amd import binding, prompt
    prompt.lib()
    return prompt, binding


def _plan(lib, c, **over):
    prompt, binding = lib
    d = dict(n_q_heads=c.heads, n_kv_heads=c.kv_heads, head_dim=c.head_dim, dtype=binding.BF16 if c.dtype == BF else binding.F32,
             max_batch=len(c.sizes), max_new=max(len(c.q), 1), max_kv_len=c.max_kv, device="cuda:0")
    d.update(over)
    return prompt.ChunkPlan(**d)


def _cache(c, rows_first=False):
    """The cache on the GPU, [page][head][row][D] or as a view of [page][row][head][D]."""
    def put(t):
        return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if rows_first else t.cuda()
    return put(c.k_pages), put(c.v_pages), c.table.cuda(), c.off.cuda(), c.kv_len.cuda()


def _attend(lib, c, plan=None, guard=2, rows_first=False, fused=False, scale=None, status=True):
    """Output rows of the batch's tokens; `guard` rows behind them have to stay as they were."""
    plan = plan or _plan(lib, c, max_new=len(c.q) + guard)
    q = torch.cat([c.q, torch.ones(guard, c.heads, c.head_dim, dtype=c.dtype)]).cuda()
    if fused:
        wide = torch.full((len(q), c.heads + 2 * c.kv_heads, c.head_dim), math.nan, dtype=c.dtype, device="cuda")
        wide[:, :c.heads] = q
        q = wide[:, :c.heads]
    out = torch.full((len(q), c.heads, c.head_dim), 77.0, dtype=c.dtype, device="cuda")
    st = torch.full((len(c.sizes),), -9, dtype=torch.int32, device="cuda") if status else None
    plan.attend(q, *_cache(c, rows_first), out, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv, scale=scale,
                status=st)
    torch.cuda.synchronize()
    if status:
        assert st.tolist() == [0] * len(c.sizes)
    assert bool((out[len(c.q):] == 77.0).all())
    return out[:len(c.q)].cpu()


def _close(got, want, tol):
    got = got.to(pc.F64)
    assert torch.equal(got.isnan(), want.isnan())
    off = torch.where(want.isnan() | (got == want), 0.0, (got - want).abs() / tol)
    assert float(off.max() if off.numel() else 0) <= 1.0, f"off by {float(off.max())} of the tolerance"


SIZES = {
    "one": [(1, 0)],
    "two-rows": [(1, 1)],
    "decode": [(1, 31), (1, 32), (1, 33), (1, 0), (1, 700)],
    "chunk": [(37, 91)],
    "prompt": [(130, 0)],
    "mixed": [(1, 500), (0, 40), (65, 3), (64, 64), (0, 0), (1, 63), (17, 127), (2, 1)],
}


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", [
    (BF, 8, 2, 64, 16), (BF, 4, 4, 128, 24), (BF, 14, 2, 128, 64), (BF, 3, 1, 64, 7), (BF, 16, 1, 128, 1),
    (BF, 5, 5, 64, 1000), (F32, 4, 4, 64, 16), (F32, 6, 2, 128, 9), (F32, 2, 1, 64, 1000),
])
def test_attention(lib, name, dtype, heads, kv_heads, head_dim, page):
    c = pc.make(SIZES[name], dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, seed=len(name))
    _close(_attend(lib, c), *pc.attention(c))


@pytest.mark.parametrize("dtype,sizes,kv_heads,group,head_dim,page", [
    (BF, [(1, 9000)], 2, 4, 128, 16),            # one token, the cache in many splits
    (BF, [(1, 5000), (1, 20), (1, 2600)], 1, 7, 64, 24),
    (BF, [(33, 4000)], 1, 8, 128, 64),           # 264 rows per head over splits
    (BF, [(300, 1000), (1, 3000), (40, 0)], 2, 1, 64, 48),
    (BF, [(700, 0)], 1, 2, 128, 700),            # several row blocks, one page
    (BF, [(4, 2049), (5, 2047)], 4, 4, 128, 33),
    (BF, [(300, 1000), (1, 3000), (40, 0), (9, 2500)], 2, 4, 128, 16),   # both kinds in one launch, joined
    (BF, [(16, 1500), (9, 70), (1, 129)], 2, 4, 64, 16),                 # up to 64 rows per head
    (BF, [(8, 1500), (5, 4000)], 1, 8, 128, 40),
    (BF, [(2, 6000)], 3, 16, 128, 128),          # 32 rows per head
    (F32, [(1, 5000)], 2, 2, 64, 16),
    (F32, [(90, 2000), (1, 100)], 1, 3, 128, 20),
])
def test_attention_long(lib, dtype, sizes, kv_heads, group, head_dim, page):
    c = pc.make(sizes, dtype=dtype, heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page=page, seed=7)
    _close(_attend(lib, c), *pc.attention(c))


@pytest.mark.parametrize("dtype,head_dim", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("step", [32, 128])
def test_numbers_of_splits(lib, dtype, head_dim, step):
    """One token over 2 to 4, 16, 17 and 64 splits of either size, alone and beside a short sequence."""
    for n in (2, 3, 4, 5, 16, 17, 64):
        for more in ([], [(3, 40)]):
            c = pc.make([(1, n * step - 1)] + more, dtype=dtype, heads=6, kv_heads=2, head_dim=head_dim, page=32, seed=n)
            _close(_attend(lib, c), *pc.attention(c))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_strides_and_scale(lib, dtype):
    """Queries as a slice of a wider projection, a cache with rows before heads, a scale of the caller's."""
    c = pc.make([(3, 100), (20, 30)], dtype=dtype, heads=8, kv_heads=4, head_dim=64, page=16, seed=3)
    want = pc.attention(c, scale=0.3)
    _close(_attend(lib, c, rows_first=True, fused=True, scale=0.3, status=False), *want)


def test_attention_in_place(lib):
    """The output over the queries, also where splits are joined."""
    c = pc.make([(1, 3000), (9, 40)], heads=4, kv_heads=2, head_dim=128, page=32, seed=4)
    q = c.q.cuda()
    _plan(lib, c).attend(q, *_cache(c), q, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv)
    _close(q.cpu(), *pc.attention(c))


@pytest.mark.parametrize("dtype,head_dim", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("sizes", [[(40, 25)], [(300, 10)], [(9, 1500)], [(20, 30)]])
def test_rows_not_seen_have_no_part(lib, dtype, head_dim, sizes):
    """A new token's NaN or infinite key and value reach the tokens from it on, and none before."""
    c = pc.make(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=head_dim, page=16, seed=5)
    n, l = sizes[0]
    kr, vr = c.rows[0]
    for i, (kind, value) in {n - 1: ("v", math.inf), n - 2: ("k", math.nan), n // 2: ("v", -math.inf),
                             n // 2 + 1: ("v", math.nan)}.items():
        r = l + i
        (vr if kind == "v" else kr)[r, 1, 5 if kind == "v" else 0] = value
        (c.v_pages if kind == "v" else c.k_pages)[c.table[0, r // 16], 1, r % 16] = (vr if kind == "v" else kr)[r, 1]
    want, tol = pc.attention(c)
    assert bool(want[: n // 2].isfinite().all()) and not bool(want[n // 2:].isfinite().all())
    got = _attend(lib, c)
    _close(got[: n // 2], want[: n // 2], tol[: n // 2])
    clean = torch.where(want[n // 2:n - 2].isfinite(), 1.0, 0.0).bool()
    _close(torch.where(clean, got[n // 2:n - 2], 0.0), torch.where(clean, want[n // 2:n - 2], 0.0), tol[n // 2:n - 2].nan_to_num(1.0))
    assert not bool(got[n // 2:n - 2].to(pc.F64)[~clean].isfinite().any())
    assert bool(got[n - 2:, 2:].isnan().all())  # a NaN score


@pytest.mark.parametrize("low", ["min", "-inf-like"])
def test_scores_of_the_lowest_values(lib, low):
    """Scores spread over hundreds of units, and scores at which every weight but one vanishes."""
    c = pc.make([(5, 60)], dtype=F32, heads=2, kv_heads=1, head_dim=64, page=16, seed=6)
    c.q *= 40.0 if low == "min" else 400.0
    _close(_attend(lib, c), *pc.attention(c))


def _append(lib, c, fused=False, rows_first=False, guard=0):
    k, v = c.k_new, c.v_new
    if guard:
        k, v = (torch.cat([t, torch.full((guard, *t.shape[1:]), 9.0, dtype=t.dtype)]) for t in (k, v))
    k, v = k.cuda(), v.cuda()
    if fused:
        wide = torch.cat([torch.zeros(len(k), c.heads, c.head_dim, dtype=c.dtype, device="cuda"), k, v], 1)
        k, v = wide[:, c.heads:c.heads + c.kv_heads], wide[:, c.heads + c.kv_heads:].clone()
    kp, vp, table, off, kv_len = _cache(c, rows_first)
    st = torch.full((len(c.sizes),), -9, dtype=torch.int32, device="cuda")
    plan = _plan(lib, c, max_new=len(k) or 1)
    plan.append(k, v, kp, vp, table, off, kv_len, max_new_in_batch=c.max_new, status=st)
    torch.cuda.synchronize()
    return kp.cpu(), vp.cpu(), st.tolist()


@pytest.mark.parametrize("name", sorted(SIZES))
@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page", [
    (BF, 8, 2, 64, 16), (BF, 4, 4, 128, 24), (F32, 3, 3, 128, 1), (F32, 20, 20, 64, 1000), (BF, 70, 70, 128, 5)])
def test_append(lib, name, dtype, heads, kv_heads, head_dim, page):
    c = pc.make(SIZES[name], dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, stale=3.0, seed=1)
    want_k, want_v = c.k_pages.clone(), c.v_pages.clone()
    for b, (n, l) in enumerate(c.sizes):  # the new rows are not there yet
        for r in range(l, l + n):
            for t in (c.k_pages, c.v_pages):
                t[c.table[b, r // page], :, r % page] = -5.0
    for fused, rows_first, guard in ((False, False, 0), (True, True, 3)):
        k, v, st = _append(lib, c, fused, rows_first, guard)
        assert st == [0] * len(c.sizes)
        assert torch.equal(k, want_k) and torch.equal(v, want_v)


@pytest.mark.parametrize("longest", [0, 70])
def test_many_sequences(lib, longest):
    """More sequences than a wave has lanes, many of them empty; with longer chunks among them."""
    sizes = [((b * 7) % 4, (b * 13) % 50) for b in range(150)]
    if longest:
        sizes[3], sizes[100] = (longest, 200), (longest - 3, 0)
    c = pc.make(sizes, heads=2, kv_heads=1, head_dim=64, page=16, seed=2, stale=0.0)
    _close(_attend(lib, c), *pc.attention(c))
    k, v, st = _append(lib, c)
    assert st == [0] * 150 and torch.equal(k, c.k_pages) and torch.equal(v, c.v_pages)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_bad_sequences_are_reported_and_leave_the_others_alone(lib, dtype):
    """Negative and too large lengths, decreasing offsets, page ids out of range."""
    sizes = [(3, 20), (2, 30), (4, 10), (1, 33), (5, 17), (2, 2)]
    c = pc.make(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=64, page=16, seed=8, spare=0, stale=0.0)
    want, tol = pc.attention(c)
    c.kv_len[1] = -1
    c.kv_len[3] = 10 ** 6                      # above what the call says
    c.table[2, 0] = 10 ** 6
    c.table[4, 1] = -7
    c.off[6] = c.off[5] - 1                    # the last sequence's end is before its start
    st = torch.zeros(6, dtype=torch.int32, device="cuda")
    out = torch.zeros(len(c.q), 4, 64, dtype=dtype, device="cuda")
    plan = _plan(lib, c, max_kv_len=40)
    kp, vp, table, off, kv_len = _cache(c)
    plan.attend(c.q.cuda(), kp, vp, table, off, kv_len, out, max_new_in_batch=5, max_kv_len_in_batch=40, status=st)
    assert st.tolist() == [0, 6, 11, 6, 11, 2]
    _close(out[:3].cpu(), want[:3], tol[:3])
    before = kp.clone()
    st.zero_()
    plan.append(c.k_new.cuda(), c.v_new.cuda(), kp, vp, table, off, kv_len, max_new_in_batch=5, max_kv_len_in_batch=40,
                status=st)
    # (sequence 2 appends rows 10-13, of its bad page; sequence 4 rows 17-21, of its bad page)
    assert st.tolist() == [0, 6, 11, 6, 11, 2]
    assert torch.equal(kp, before)  # sequence 0's rows were there already
    # too few tokens per sequence, then offsets past the packed rows
    plan.attend(c.q.cuda(), kp, vp, table, off, kv_len, out, max_new_in_batch=2, max_kv_len_in_batch=40, status=st)
    assert st.tolist()[0] == 2
    plan.attend(c.q[:4].cuda(), kp, vp, table, off, kv_len, out[:4], max_new_in_batch=3, max_kv_len_in_batch=40, status=st)
    assert st.tolist()[:2] == [0, 2]


def test_offsets_past_32_bits(lib):
    """A cache of more than 2^32 bytes, read and written behind that."""
    prompt, binding = lib
    page, d, n_pages = 64, 128, 150_000   # 64 * 128 * 2 bytes each, 2.4 GB per tensor; strides of two
    k = torch.zeros(n_pages, 2, 1, page, d, dtype=BF, device="cuda")[:, 0]
    v = torch.zeros(n_pages, 2, 1, page, d, dtype=BF, device="cuda")[:, 0]
    assert (n_pages - 1) * k.stride(0) * 2 > 2 ** 32
    c = pc.make([(3, 190)], heads=4, kv_heads=1, head_dim=d, page=page, seed=9, stale=0.0)
    ids = torch.tensor([n_pages - 1, 140_000, 3, n_pages - 2], dtype=torch.int32)
    for j in range(4):
        k[ids[j].item()], v[ids[j].item()] = c.k_pages[c.table[0, j]].cuda(), c.v_pages[c.table[0, j]].cuda()
    k[ids[3].item()], v[ids[3].item()], k[3, :, 62:], v[3, :, 62:], k[ids[2].item(), :, 62:] = 0, 0, 0, 0, 0
    plan = _plan(lib, c)
    off, kv_len, table = c.off.cuda(), c.kv_len.cuda(), ids[None].cuda()
    plan.append(c.k_new.cuda(), c.v_new.cuda(), k, v, table, off, kv_len, max_new_in_batch=3)
    out = torch.empty(3, 4, d, dtype=BF, device="cuda")
    plan.attend(c.q.cuda(), k, v, table, off, kv_len, out, max_new_in_batch=3, max_kv_len_in_batch=190)
    _close(out.cpu(), *pc.attention(c))


# ---------------------------------------------------------------------------
# scores
# ---------------------------------------------------------------------------

def _score(lib, z, token, topk, only=None):
    prompt, binding = lib
    plan = prompt.ScorePlan(vocab=z.shape[1], max_rows=max(len(z), 1), topk_out=topk,
                            dtype=binding.BF16 if z.dtype == BF else binding.F32, device="cuda:0")
    out = prompt.alloc_score_outputs(rows=len(z), topk_out=topk, device="cuda:0")
    for t in out.values():
        t.fill_(-77)
    plan.score(z, token.cuda() if token is not None else None, {k: v for k, v in out.items() if only is None or k in only})
    torch.cuda.synchronize()
    return {k: v.cpu() for k, v in out.items()}


def _check_scores(got, z, token, topk):
    want, tol = pc.score(z, token, topk)
    for k in want:
        if k in tol:
            _close(got[k], want[k], tol[k])
        else:
            assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("vocab,rows,topk", [(1, 3, 1), (5, 2, 5), (16, 1, 16), (100, 4, 8), (255, 3, 16), (1003, 5, 5),
                                             (2049, 2, 8), (9001, 1, 16), (32000, 1, 8), (50257, 3, 8), (8192, 1100, 8),
                                             (152064, 2, 16)])
def test_scores(lib, dtype, vocab, rows, topk):
    gen = torch.Generator().manual_seed(vocab + topk)
    z = (torch.randn(rows, vocab, generator=gen) * 3).to(dtype)
    token = torch.randint(vocab, (rows,), generator=gen).int()
    token[0] = int(z[0].float().argmax())
    _check_scores(_score(lib, z.cuda(), token, topk), z, token, topk)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (5, 2), (8, 7)])
def test_scores_of_rows_at_any_alignment(lib, dtype, pad, shift):
    gen = torch.Generator().manual_seed(pad * 10 + shift)
    for vocab in (3, 7, 8, 9, 777, 4100):
        flat = torch.full((shift + 6 * (vocab + pad),), math.nan, dtype=dtype)
        rows = flat[shift:].view(6, vocab + pad)
        z = (torch.randn(6, vocab, generator=gen) * 3).to(dtype)
        rows[:, :vocab] = z
        token = torch.randint(vocab, (6,), generator=gen).int()
        token[1], token[2] = 0, vocab - 1
        dev = flat.cuda()[shift:].view(6, vocab + pad)[:, :vocab]
        _check_scores(_score(lib, dev, token, 3), z, token, 3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("vocab", [40, 5000, 20011])
def test_scores_of_odd_rows(lib, dtype, vocab):
    """Masked vocabularies, ties, orders, values that are not numbers, tokens that are none."""
    inf, lowest = math.inf, torch.finfo(dtype).min
    gen = torch.Generator().manual_seed(vocab)
    base = (torch.randn(vocab, generator=gen) * 2).to(dtype)
    ids = torch.arange(vocab)
    few = torch.where(ids % 13 == 5, base, -inf)                       # a masked vocabulary
    one = torch.where(ids == vocab - 2, base, -inf)
    low = torch.where(ids % 2 == 0, base, lowest)                      # masked by the lowest value
    rows = [torch.full((vocab,), -inf), few, one, low, torch.full((vocab,), lowest), torch.zeros(vocab),
            torch.where(ids % 2 == 0, 0.0, -0.0), torch.full((vocab,), 2.5), ids.float() / 64, -ids.float() / 64,
            (ids % 3).float(), (ids * 7 % 256 < 9).float() * 4 + ids.float() / 1024, torch.where(ids == 3, math.nan, base),
            torch.where(ids == vocab - 1, inf, base), torch.full((vocab,), math.nan), base * 30, base, base, base]
    z = torch.stack([r.to(dtype) for r in rows])
    token = torch.full((len(rows),), 7, dtype=torch.int32)
    token[2] = vocab - 2
    token[-3], token[-2], token[-1] = -1, vocab, -5
    for topk in (5, 16):
        _check_scores(_score(lib, z.cuda(), token, topk), z, token, topk)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_where_few_threads_hold_the_largest(lib, dtype):
    """The largest logits at distances that put them all into few threads' vectors, more than are kept at once."""
    n = 8 if dtype == BF else 4
    vocab = 256 * n * 40
    ids = torch.arange(vocab)
    lane = (ids // n) % 256
    z = torch.where(lane < 12, 50.0 - (ids % 97).float() / 4, -5.0)[None].repeat(700, 1).to(dtype)
    token = (ids[:700] * 37 % vocab).int()
    _check_scores(_score(lib, z.cuda(), token, 16), z, token, 16)


def test_scores_written_as_asked(lib):
    """Outputs that are not asked for stay as they were; no tokens at all."""
    z = torch.randn(3, 100)
    got = _score(lib, z.cuda(), None, 4, only=("entropy",))
    want, tol = pc.score(z, torch.full((3,), -1), 4)
    _close(got["entropy"], want["entropy"], tol["entropy"])
    assert all(bool((v == -77).all()) for k, v in got.items() if k != "entropy")
    got = _score(lib, z.cuda(), None, 4)
    assert got["tok_logprob"].tolist() == [0.0] * 3 and got["tok_rank"].tolist() == [-1] * 3


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def _chain(lib, c, w, cache, plan, score, out, results, tokens):
    """The new tokens through cache, attention, LM head and scores."""
    kp, vp, table, off, kv_len = cache
    plan.append(c["k_new"], c["v_new"], kp, vp, table, off, kv_len, max_new_in_batch=len(c["q"]))
    plan.attend(c["q"], kp, vp, table, off, kv_len, out, max_new_in_batch=len(c["q"]), max_kv_len_in_batch=300)
    logits = (c["q"] + out).flatten(1).float() @ w
    score.score(logits, tokens, results)


def test_captured_chain_replays(lib):
    """Append, attention and scores captured once, replayed with other lengths and eager work in between."""
    prompt, binding = lib
    c = pc.make([(5, 150), (1, 300), (0, 7), (3, 64)], heads=4, kv_heads=2, head_dim=64, page=16, seed=12, stale=0.0, spare=20)
    used = c.table[c.table >= 0]
    free = [x for x in range(len(c.k_pages)) if x not in set(used.tolist())]
    c.table[c.table < 0] = free[0]   # room for longer sequences (their rows there are shared and never read apart)
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn(256, 500, generator=gen, device="cuda") * 0.2
    x = {k: getattr(c, k).cuda() for k in ("q", "k_new", "v_new")}
    tokens = torch.arange(len(c.q), dtype=torch.int32, device="cuda") * 50
    plan, score = _plan(lib, c, max_kv_len=300), prompt.ScorePlan(vocab=500, max_rows=len(c.q), device="cuda:0")

    def buffers():
        return _cache(c), torch.zeros(len(c.q), 4, 64, dtype=BF, device="cuda"), prompt.alloc_score_outputs(
            rows=len(c.q), topk_out=8)

    cache, out, results = buffers()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _chain(lib, x, w, cache, plan, score, out, results, tokens)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        _chain(lib, x, w, cache, plan, score, out, results, tokens)
    for k, (off, lens) in enumerate([([0, 5, 6, 6, 9], [150, 300, 7, 64]), ([0, 1, 2, 4, 5], [3, 299, 0, 80]),
                                     ([0, 5, 6, 6, 9], [150, 300, 7, 64]), ([2, 2, 3, 3, 9], [10, 160, 7, 5])]):
        for t, v in ((cache[3], off), (cache[4], lens)):
            t.copy_(torch.tensor(v, dtype=torch.int32))
        for v in x.values():
            v.normal_(generator=gen)
        e_cache, e_out, e_results = buffers()
        e_cache[0].copy_(cache[0]), e_cache[1].copy_(cache[1])
        e_cache[3].copy_(cache[3]), e_cache[4].copy_(cache[4])
        e_out.copy_(out)
        graph.replay()
        torch.cuda.synchronize()
        e_plan = _plan(lib, c, max_kv_len=300)
        _chain(lib, x, w, e_cache, e_plan, prompt.ScorePlan(vocab=500, max_rows=len(c.q), device="cuda:0"), e_out, e_results, tokens)
        torch.cuda.synchronize()
        lo, hi = off[0], off[-1]
        assert torch.equal(out[lo:hi], e_out[lo:hi]), k
        assert torch.equal(cache[0], e_cache[0]) and torch.equal(cache[1], e_cache[1])
        for name in results:
            assert torch.equal(results[name][lo:hi], e_results[name][lo:hi]), (k, name)


def test_nothing_to_do(lib):
    """No sequences, and sequences without tokens: nothing is written but their status."""
    for sizes in ([], [(0, 5), (0, 0)]):
        c = pc.make(sizes, heads=4, kv_heads=2, head_dim=64, page=16)
        plan = _plan(lib, c, max_batch=2, max_new=4, max_kv_len=10)
        st = torch.full((len(sizes),), -9, dtype=torch.int32, device="cuda")
        out = torch.full((4, 4, 64), 7.0, dtype=BF, device="cuda")
        cache = _cache(c)
        before = cache[0].clone()
        kw = dict(max_new_in_batch=0, status=st)
        plan.attend(out[:0], *cache, out[:0], max_kv_len_in_batch=10, **kw)
        assert st.tolist() == [0] * len(sizes)
        st.fill_(-9)
        plan.append(c.k_new.cuda(), c.v_new.cuda(), *cache, **kw)
        assert st.tolist() == [0] * len(sizes) and bool((out == 7.0).all())
        assert torch.equal(cache[0].nan_to_num(3.0), before.nan_to_num(3.0))
    prompt, binding = lib
    score = prompt.ScorePlan(vocab=100, max_rows=4, device="cuda:0")
    score.score(torch.zeros(0, 100, device="cuda"), None, prompt.alloc_score_outputs(rows=0, topk_out=8))


def test_two_plans_at_once(lib):
    """Calls that overlap on two streams, a workspace each."""
    cases = [pc.make([(1, 4000), (70, 600)], heads=8, kv_heads=2, head_dim=d, page=16, seed=20 + d) for d in (64, 128)]
    runs = []
    for c in cases:
        q = c.q.cuda()
        runs.append((_plan(lib, c), q, _cache(c), torch.empty_like(q), torch.cuda.Stream(), c))
    torch.cuda.synchronize()
    for _ in range(20):
        for plan, q, cache, out, stream, c in runs:
            plan.attend(q, *cache, out, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv, stream=stream)
    torch.cuda.synchronize()
    for plan, q, cache, out, stream, c in runs:
        _close(out.cpu(), *pc.attention(c))


def test_results_repeat_on_another_stream(lib):
    """The same call on a stream of its own, and again: bit for bit."""
    c = pc.make([(70, 900), (1, 4000), (3, 10)], heads=8, kv_heads=2, head_dim=128, page=16, seed=13)
    plan = _plan(lib, c)
    cache, q = _cache(c), c.q.cuda()
    outs = [torch.empty_like(q) for _ in range(3)]
    kw = dict(max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv)
    plan.attend(q, *cache, outs[0], **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    plan.attend(q, *cache, outs[1], **kw, stream=side)
    side.synchronize()
    with torch.cuda.stream(side):
        plan.attend(q, *cache, outs[2], **kw)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_prompt_then_verification(lib):
    """A prompt goes through append, attention and scores in two chunks, over the verification step's own cache:
    its entropies and logits are those of root-only verification steps, token by token, and the
    drafting session triggers on them."""
    import numpy as np
    import decode_loop
    from paper_2511_01282_amd import draft, runner
    prompt, binding = lib
    m = decode_loop.make_model(n_heads=4, head_dim=64, hidden=256)
    s = m.shape
    text = decode_loop.prompt(n=48)
    T, cap = len(text), 64
    k_cache = torch.zeros(1, s.n_kv_heads, cap, s.head_dim, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    plan = prompt.ChunkPlan(n_q_heads=4, n_kv_heads=s.n_kv_heads, head_dim=64, dtype=binding.F32, max_batch=1, max_new=40,
                            max_kv_len=cap, device="cuda:0")
    score = prompt.ScorePlan(vocab=s.vocab, max_rows=T, topk_out=8, device="cuda:0")
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")   # one page: the sequence's rows
    h = torch.from_numpy(m.E_h[text]).cuda()
    k, v = (torch.from_numpy(t[text]).cuda().view(T, s.n_kv_heads, 64) for t in (m.E_k, m.E_v))
    out = torch.empty(T, 4, 64, device="cuda")
    for lo, hi in ((0, 31), (31, T)):
        off = torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda")
        kv_len = torch.tensor([lo], dtype=torch.int32, device="cuda")
        plan.append(k[lo:hi], v[lo:hi], k_cache, v_cache, table, off, kv_len, max_new_in_batch=hi - lo)
        plan.attend(h[lo:hi].view(-1, 4, 64), k_cache, v_cache, table, off, kv_len, out[lo:hi], max_new_in_batch=hi - lo,
                    max_kv_len_in_batch=lo)
    logits = (h + out.view(T, -1)) @ torch.from_numpy(m.W).cuda().T.contiguous()
    token = torch.tensor(list(text[1:]) + [-1], dtype=torch.int32, device="cuda")
    got = prompt.alloc_score_outputs(rows=T, topk_out=8)
    score.score(logits, token, got)
    for t in (0, 1, 5, 30, 31, 47):
        w = decode_loop.workload(m, text[:t + 1], [-1], [int(text[t])], [0])
        ref = runner.run(w, device="cuda:0")
        # the same sums in float32 in another order
        np.testing.assert_allclose(out[t].flatten().cpu(), ref["attn_out"][0], rtol=2e-5, atol=2e-5)
        np.testing.assert_allclose(got["entropy"][t].item(), ref["entropy"][0], rtol=1e-4, atol=1e-4)
        np.testing.assert_allclose(got["lse"][t].item(), ref["lse"][0], rtol=1e-4, atol=1e-4)
        assert int(got["topk_id"][t, 0]) == int(ref["argmax"][0])
    # a verification step on the very cache: rows 0..T-2 are the prefix, row T-1 the root's own
    w = decode_loop.workload(m, text, [-1], [int(text[-1])], [0])
    ref = runner.run(w, device="cuda:0")
    ins = runner.upload(w, "cuda:0")
    ins["k_cache"], ins["v_cache"] = k_cache, v_cache
    w.k_cache = np.zeros((1, s.n_kv_heads, cap, 64), np.float32)
    same = runner.run(w, inputs=ins, device="cuda:0")
    np.testing.assert_array_equal(same["argmax"], ref["argmax"])
    np.testing.assert_allclose(same["logits"], ref["logits"], rtol=1e-5, atol=1e-5)
    # the prompt's entropies: token t was drawn from the distribution at t - 1
    ent = np.concatenate([[np.nan], got["entropy"][:-1].cpu().numpy()]).astype(np.float32)
    session = draft.DraftSession()
    session.append(text, ent)
    trigger = draft.trigger_eval(ent)
    assert trigger.key_len >= 1 and session.propose().trigger == trigger
    blind = draft.DraftSession()
    blind.append(text, None)
    assert blind.propose().trigger.key_len == 0
