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
