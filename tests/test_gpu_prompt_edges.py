"""The prompt side on the GPU at the ends of what its interface allows, against the operators in 64 bits
(tests/prompt_cases.py)."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import prompt_cases as pc  # noqa: E402
from test_gpu_prompt import BF, F32, _check_scores, _close, _score, lib  # noqa: E402,F401


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
