"""The prompt side on the host at the ends of what its interface allows: no call here reaches the GPU (see
test_prompt_host.py)."""
import ctypes

import pytest

from test_prompt_host import FAKE, OK, _batch, _chunk_shape, _create, p  # noqa: F401


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
