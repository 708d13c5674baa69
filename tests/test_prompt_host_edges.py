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
