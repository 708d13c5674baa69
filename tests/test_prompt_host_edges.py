"""The prompt side on the host at the ends of what its interface allows: no call here reaches the GPU (see
test_prompt_host.py)."""
import ctypes

import pytest

from test_prompt_host import FAKE, OK, SHAPE, _batch, _chunk_shape, _create, p  # noqa: F401


@pytest.mark.parametrize("dtype,heads", [(0, 8), (1, 8), (1, 64)])
@pytest.mark.parametrize("total", [0, 5])
def test_no_tokens_in_any_sequence(p, dtype, heads, total):
    """Nothing to compute and no status to report: nothing is launched, whatever rows there are."""
    st, h = _create(p, "chunk", _chunk_shape(p, dtype=dtype, n_q_heads=heads))
    assert st == OK
    a = p.AttnArgs(_batch(p, total_new=total, max_new_in_batch=0), FAKE, 512, 64, FAKE, 512, 64, 0.0)
    assert p.lib().respec_chunk_attn(h, ctypes.byref(a), FAKE, None) == OK
    p.lib().respec_chunk_destroy(h)


@pytest.mark.parametrize("scale", [0.0, -1.0, 1e-50, float("nan")])
def test_binding_refuses_scales_that_are_not_positive(p, scale):
    """... in float32, as which they are passed: one that rounds to 0 would stand for the default."""
    import torch
    plan = p.ChunkPlan(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=1, max_batch=2, max_new=8, max_kv_len=64, device="cpu")
    bf, i32 = torch.bfloat16, torch.int32
    q, pages = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(5, 2, 16, 64, dtype=bf)
    with pytest.raises(ValueError):
        plan.attend(q, pages, pages, torch.zeros(1, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32), q,
                    max_new_in_batch=3, max_kv_len_in_batch=9, scale=scale)


@pytest.mark.parametrize("kind,shape,batch", [
    # 2^28 tokens of one head of 64 columns, 16 to a workgroup of 256 threads
    ("append", dict(n_q_heads=1, n_kv_heads=1, max_new=1 << 28), dict(batch=1, total_new=1 << 28, max_new_in_batch=1)),
    # a workgroup per sequence and KV head, and one per sequence's status
    ("attn", dict(n_q_heads=256, n_kv_heads=256, max_batch=65535, max_new=65535, dtype=1),
     dict(batch=65535, total_new=65535, max_new_in_batch=1, seq_status=FAKE)),
    ("attn", dict(n_q_heads=256, n_kv_heads=256, max_batch=65535, max_new=65535, dtype=0),
     dict(batch=65535, total_new=65535, max_new_in_batch=1, seq_status=FAKE)),
    # blocks of 256 query rows, 512 threads each; of 64, 256 threads
    ("attn", dict(n_q_heads=256, n_kv_heads=256, max_new=(1 << 23) - 1, dtype=1),
     dict(batch=1, total_new=(1 << 23) - 1, max_new_in_batch=(1 << 23) - 1)),
    ("attn", dict(n_q_heads=64, n_kv_heads=64, max_new=1 << 24, dtype=0),
     dict(batch=1, total_new=1 << 24, max_new_in_batch=1 << 24)),
])
def test_launches_of_too_many_threads(p, kind, shape, batch):
    """A dispatch counts its threads in 32 bits: refused by the host, not by the launch."""
    st, h = _create(p, "chunk", _chunk_shape(p, **shape))
    assert st == OK
    b = _batch(p, **dict(batch, max_kv_len_in_batch=0))
    if kind == "append":
        a = p.AppendArgs(b, FAKE, FAKE, 0, 0, 0, 0)
        assert p.lib().respec_chunk_append(h, ctypes.byref(a), None) == SHAPE
    else:
        a = p.AttnArgs(b, FAKE, 0, 0, FAKE, 0, 0, 0.0)
        assert p.lib().respec_chunk_attn(h, ctypes.byref(a), FAKE, None) == SHAPE
    p.lib().respec_chunk_destroy(h)


@pytest.mark.parametrize("rows,status", [((1 << 24) - 1, OK), (1 << 24, SHAPE), (2**31 - 1, SHAPE)])
def test_rows_of_a_score_plan(p, rows, status):
    st, h = _create(p, "score", p.ScoreShape(100, 0, rows, 8))
    assert st == status
    p.lib().respec_score_destroy(h)
