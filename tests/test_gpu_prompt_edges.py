"""The prompt side on the GPU at the ends of what its interface allows, against the operators in 64 bits
(tests/prompt_cases.py)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import prompt_cases as pc  # noqa: E402
from test_gpu_prompt import BF, F32, _attend, _cache, _check_scores, _close, _plan, _score, lib  # noqa: E402,F401


# ---------------------------------------------------------------------------
# scores
# ---------------------------------------------------------------------------

def _masked_rows(vocab, dtype, low, gen):
    """Rows of which most logits are `low`, and a token that is not."""
    ids = torch.arange(vocab)
    some = torch.randperm(vocab, generator=gen)[:20]
    keep = [torch.isin(ids, some), ids >= vocab - 11, ids < 50, ids == vocab // 2, ids % 13 == 5,
            (ids > vocab // 3) & (ids < 2 * vocab // 3), (ids < 3) | (ids >= vocab - 3), ids // 64 % 9 == 4]
    z = (torch.randn(len(keep), vocab, generator=gen) * 3).to(dtype)
    z = torch.where(torch.stack(keep), z, torch.full((), low).to(dtype))
    return z, torch.tensor([int(k.nonzero()[-1]) for k in keep], dtype=torch.int32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("low", ["min", -1e38, -1e37, -1e30])
@pytest.mark.parametrize("vocab", [700, 20011, 152064])
def test_scores_of_rows_masked_by_a_low_value(lib, dtype, low, vocab):
    """Finite logits have finite statistics: threads, waves and parts of a row that saw masked logits alone."""
    gen = torch.Generator().manual_seed(vocab)
    z, token = _masked_rows(vocab, dtype, torch.finfo(dtype).min if low == "min" else low, gen)
    got = _score(lib, z.cuda(), token, 8)          # a few rows: in parts
    _check_scores(got, z, token, 8)
    times = 520 // len(z) + 1                      # many: a workgroup each
    many = _score(lib, z.repeat(times, 1).cuda(), token.repeat(times), 8)
    want, tol = pc.score(z, token, 8)
    for k in want:
        for i in range(times):
            part = many[k][i * len(z):(i + 1) * len(z)]
            if k in tol:
                _close(part, want[k], tol[k])
            else:
                assert torch.equal(part, want[k]), k


def test_scores_behind_32_bits(lib):
    """Rows whose logits lie past 2^32 bytes."""
    gen = torch.Generator().manual_seed(1)
    stride = (1 << 26) + 3
    flat = torch.empty(36, stride, dtype=BF, device="cuda")
    z = (torch.randn(36, 5000, generator=gen) * 3).to(BF)
    flat[:, :5000] = z.cuda()
    token = torch.randint(5000, (36,), generator=gen).int()
    assert 35 * stride * 2 > 2 ** 32
    _check_scores(_score(lib, flat[:, :5000], token, 5), z, token, 5)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,head_dim", [(BF, 64), (BF, 128), (F32, 64)])
@pytest.mark.parametrize("sizes", [[(1, 0)], [(1, 200)], [(1, 5000)], [(20, 900)], [(150, 40)], [(40, 2000), (1, 300)]])
@pytest.mark.parametrize("score", [-3.2e38, -1e30, 2.5e9, -4e12, 3.1e38])
def test_scores_of_any_finite_size(lib, dtype, head_dim, sizes, score):
    """Keys all alike have weights all alike, however large the scores are.

    A token's output is the mean of the values it sees.  The weights of equal scores are equal, so neither their size
    nor their rounding matters; the sums add (rows + 64) 2^-24, the result's rounding half a step."""
    c = pc.make(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=head_dim, page=16, seed=3, stale=0.0)
    big = math.sqrt(abs(score) / math.log2(math.e) / (head_dim / 2))
    c.q[:] = 0
    c.k_pages[:] = 0
    c.q[..., ::2] = big
    c.k_pages[..., ::2] = math.copysign(big, score)   # scale 1: half of the columns have a product each
    assert math.log2(math.e) * float((c.q[0, 0].double() * c.k_pages[0, 0, 0].double()).sum().abs()) < torch.finfo(F32).max
    want, tol = torch.empty(c.q.shape, dtype=pc.F64), torch.empty(c.q.shape, dtype=pc.F64)
    t = 0
    for (n, l), (_, vr) in zip(c.sizes, c.rows):
        for i in range(n):
            v = vr[:l + i + 1].to(pc.F64).repeat_interleave(2, 1)
            want[t], size = v.mean(0), v.abs().mean(0)
            tol[t] = size * (len(v) + 64) * 2.0 ** -24 + want[t].abs() * torch.finfo(dtype).eps / 2 + 1e-30
            t += 1
    _close(_attend(lib, c, scale=1.0), want, tol)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("status", [False, True])
def test_no_tokens_in_any_sequence(lib, dtype, status):
    """Packed rows that no sequence owns (a captured call replayed without tokens), lengths that say so."""
    c = pc.make([(0, 5), (0, 0)], dtype=dtype, heads=4, kv_heads=2, head_dim=64, page=16)
    plan = _plan(lib, c, max_new=5)
    rows = torch.full((5, 4, 64), 7.0, dtype=dtype, device="cuda")
    out = rows.clone()
    st = torch.full((2,), -9, dtype=torch.int32, device="cuda") if status else None
    cache = _cache(c)
    plan.attend(rows, *cache, out, max_new_in_batch=0, max_kv_len_in_batch=5, status=st)
    plan.append(rows[:, :2], rows[:, 2:], *cache, max_new_in_batch=0)
    torch.cuda.synchronize()
    assert torch.equal(out, rows) and (not status or st.tolist() == [0, 0])
    for t, was in zip(cache[:2], (c.k_pages, c.v_pages)):
        assert torch.equal(t.cpu().nan_to_num(3.0), was.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_of_dimensions_of_one(lib, dtype):
    """A dimension of one element has no stride to speak of: a token from a column vector, one page, one KV head."""
    c = pc.make([(1, 9)], dtype=dtype, heads=4, kv_heads=1, head_dim=64, page=16, spare=0, stale=0.0)
    c.table[:] = 0
    kr, vr = c.rows[0]
    k, v = (torch.zeros(16, 64, dtype=dtype) for _ in range(2))
    k[:10], v[:10] = kr[:, 0], vr[:, 0]
    q = c.q.cuda().as_strided((1, 4, 64), (1, 64, 1))
    new = [t.cuda().as_strided((1, 1, 64), (3, 5, 1)) for t in (c.k_new, c.v_new)]
    kp, vp = k.cuda().as_strided((1, 1, 16, 64), (3, 7, 64, 1)), v.cuda().as_strided((1, 1, 16, 64), (1024, 1024, 64, 1))
    table, off, kv_len = c.table[:, :1].cuda(), c.off.cuda(), c.kv_len.cuda()
    out = torch.zeros(4 * 64, dtype=dtype, device="cuda").as_strided((1, 4, 64), (5, 64, 1))
    plan = _plan(lib, c)
    plan.append(*new, kp, vp, table, off, kv_len, max_new_in_batch=1)
    plan.attend(q, kp, vp, table, off, kv_len, out, max_new_in_batch=1, max_kv_len_in_batch=9)
    _close(out.cpu(), *pc.attention(c))


@pytest.mark.parametrize("dtype,heads,kv_heads,sizes", [
    (BF, 256, 1, [(1, 300)]), (BF, 256, 1, [(3, 20), (1, 0)]), (BF, 96, 2, [(1, 700), (2, 65)]), (BF, 256, 256, [(1, 40), (33, 0)]),
    (F32, 256, 1, [(2, 130)]), (F32, 96, 2, [(1, 500), (4, 3)]),
])
def test_many_heads(lib, dtype, heads, kv_heads, sizes):
    c = pc.make(sizes, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=64, page=16, seed=heads)
    _close(_attend(lib, c), *pc.attention(c))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [[(1, 3000)], [(40, 30), (1, 500)], [(300, 0)]])
def test_output_as_a_slice(lib, dtype, sizes):
    """The output as columns of a wider tensor: joined splits and whole rows alike, and nothing beside them."""
    c = pc.make(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=128, page=32, seed=14)
    wide = torch.full((len(c.q), 7, 256), 5.0, dtype=dtype, device="cuda")
    out = wide[:, 2:6, 128:]
    _plan(lib, c).attend(c.q.cuda(), *_cache(c), out, max_new_in_batch=c.max_new, max_kv_len_in_batch=c.max_kv)
    _close(out.cpu(), *pc.attention(c))
    out.fill_(5.0)
    assert bool((wide == 5.0).all())


@pytest.mark.parametrize("dtype,page", [(BF, 16), (BF, 24), (F32, 16)])
@pytest.mark.parametrize("longest", [5, 90])
def test_good_sequences_behind_bad_ones(lib, dtype, page, longest):
    """Sequences with bad lengths and pages between good ones: the good ones' outputs and appended rows are theirs."""
    sizes = [(3, 20), (2, 30), (4, 10), (longest, 33), (5, 17), (2, 2), (1, 700)]
    bad = (1, 2, 4)
    c = pc.make(sizes, dtype=dtype, heads=4, kv_heads=2, head_dim=64, page=page, seed=21, spare=0, stale=2.0)
    want, tol = pc.attention(c)
    c.kv_len[1] = -1
    c.table[2, 0] = 10 ** 6
    c.kv_len[4] = 10 ** 6
    off = c.off.tolist()
    expect = [0, 6, 11, 0, 6, 0, 0]
    plan = _plan(lib, c, max_kv_len=700)
    k_want, v_want = c.k_pages.clone(), c.v_pages.clone()
    for b, (n, l) in enumerate(sizes):
        for r in range(l, l + n):   # no sequence's new rows are there yet
            for t, w in ((c.k_pages, k_want), (c.v_pages, v_want)):
                p = int(c.table[b, r // page])
                if 0 <= p < len(t):
                    t[p, :, r % page] = -5.0
                    if b in bad and not (b == 2 and r // page > 0):
                        w[p, :, r % page] = -5.0
    kp, vp, table, o, kv_len = _cache(c)
    st = torch.full((len(sizes),), -9, dtype=torch.int32, device="cuda")
    kw = dict(max_new_in_batch=c.max_new, max_kv_len_in_batch=700, status=st)
    plan.append(c.k_new.cuda(), c.v_new.cuda(), kp, vp, table, o, kv_len, **kw)
    # (sequence 2: rows 10-13, some of them in its good page where pages are short)
    assert st.tolist() == expect
    assert torch.equal(kp.cpu(), k_want) and torch.equal(vp.cpu(), v_want)
    out = torch.zeros(len(c.q), 4, 64, dtype=dtype, device="cuda")
    st.fill_(-9)
    plan.attend(c.q.cuda(), kp, vp, table, o, kv_len, out, **kw)
    assert st.tolist() == expect
    for b in range(len(sizes)):
        if b not in bad:
            s = slice(off[b], off[b + 1])
            _close(out[s].cpu(), want[s], tol[s])


# ---------------------------------------------------------------------------
# a plan's workspace
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("by_argument", [True, False])
def test_workspace_is_kept_for_a_call_on_another_stream(lib, by_argument):
    """A plan that is dropped while its call waits on another stream: its workspace goes to nobody else until then."""
    c = pc.make([(1, 4000)], heads=4, kv_heads=2, head_dim=64, page=16, seed=30)
    q, cache = c.q.cuda(), _cache(c)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    plan = _plan(lib, c)
    at, size = plan._ws_buf.data_ptr(), plan._ws_buf.numel()
    torch.cuda.synchronize()
    kw = dict(max_new_in_batch=1, max_kv_len_in_batch=4000)
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)   # some tens of milliseconds
        if not by_argument:
            plan.attend(q, *cache, out, **kw)
    if by_argument:
        plan.attend(q, *cache, out, stream=side, **kw)
    del plan
    other = torch.zeros(size, dtype=torch.uint8, device="cuda")
    assert other.data_ptr() != at
    torch.cuda.synchronize()
    assert not bool(other.any())
    _close(out.cpu(), *pc.attention(c))
