"""The C ABI of the prompt side on the host: exports, plans and refusals.

No call here reaches the GPU: each is refused by the host checks, or has nothing to do (fake
device addresses are never dereferenced on the host).
"""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
OK, NULL, SHAPE, DTYPE, PARAM, CAPACITY, WORKSPACE = 0, 1, 2, 3, 4, 6, 8


@pytest.fixture(scope="module")
def p():
    from paper_2511_01282_amd import binding, prompt
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_01282_amd import build
        build.build()
    prompt.lib()
    return prompt


def test_library_exports_every_declared_function(p):
    text = open(os.path.join(ROOT, "include", "respec_prompt.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert set(re.findall(r"\b(respec_[a-z_]+)\s*\(", text)) == set(p.EXPORTS)
    for name in p.EXPORTS:
        assert hasattr(p.lib(), name), name


def test_structs_match_the_header(p, tmp_path):
    """Sizes and offsets of the ctypes structs against a C compiler's."""
    import shutil
    import subprocess
    cc = shutil.which("gcc")
    if not cc:
        pytest.skip("no C compiler")
    names = {"respec_chunk_shape": p.ChunkShape, "respec_paged_cache": p.PagedCache, "respec_chunk_batch": p.ChunkBatch,
             "respec_chunk_append_args": p.AppendArgs, "respec_chunk_attn_args": p.AttnArgs,
             "respec_score_shape": p.ScoreShape, "respec_score_args": p.ScoreArgs}
    lines = []
    for c, s in names.items():
        lines.append(f'printf("%zu\\n", sizeof({c}));')
        lines += [f'printf("%zu\\n", offsetof({c}, {f[0]}));' for f in s._fields_]
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "respec_prompt.h"\nint main(void) {\n%s\nreturn 0;}\n' % "\n".join(lines))
    exe = str(tmp_path / "s")
    subprocess.check_call([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    got = [int(x) for x in subprocess.check_output([exe]).split()]
    want = []
    for s in names.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def _create(p, kind, shape, out=True):
    h = ctypes.c_void_p()
    st = getattr(p.lib(), f"respec_{kind}_create")(ctypes.byref(shape) if shape else None, ctypes.byref(h) if out else None)
    return st, h


def _chunk_shape(p, **over):
    d = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=1, max_batch=4, max_new=100, max_kv_len=1000)
    d.update(over)
    return p.ChunkShape(**d)


@pytest.mark.parametrize("over,status", [
    ({}, OK), ({"dtype": 2}, DTYPE), ({"head_dim": 96}, SHAPE), ({"n_q_heads": 7}, SHAPE), ({"n_kv_heads": 0}, SHAPE),
    ({"n_q_heads": 512}, SHAPE), ({"max_batch": 0}, SHAPE), ({"max_batch": 65536}, SHAPE), ({"max_new": 0}, SHAPE),
    ({"max_kv_len": -1}, SHAPE), ({"max_new": 1 << 28}, SHAPE), ({"max_kv_len": 2**30 - 99}, SHAPE),
    ({"max_kv_len": 2**30 - 100}, OK), ({"dtype": 0, "head_dim": 128, "n_kv_heads": 8}, OK),
])
def test_chunk_create(p, over, status):
    st, h = _create(p, "chunk", _chunk_shape(p, **over))
    assert st == status and bool(h.value) == (status == OK)
    if st == OK:
        assert p.lib().respec_chunk_workspace_bytes(h) > 0
    p.lib().respec_chunk_destroy(h)


def test_create_without_arguments(p):
    for kind in ("chunk", "score"):
        assert _create(p, kind, None)[0] == NULL
        getattr(p.lib(), f"respec_{kind}_destroy")(None)
        assert getattr(p.lib(), f"respec_{kind}_workspace_bytes")(None) == 0
    assert _create(p, "chunk", _chunk_shape(p), out=False)[0] == NULL
    assert _create(p, "score", p.ScoreShape(100, 0, 4, 8), out=False)[0] == NULL


def _batch(p, **over):
    cache = dict(k=FAKE, v=FAKE, n_pages=9, page_size=16, page_stride=2 * 16 * 64, head_stride=16 * 64, row_stride=64,
                 page_table=FAKE, table_width=5, table_stride=5)
    d = dict(batch=2, total_new=10, max_new_in_batch=8, max_kv_len_in_batch=40, new_off=FAKE, kv_len=FAKE, seq_status=None)
    cache.update({k: v for k, v in over.items() if k in cache})
    d.update({k: v for k, v in over.items() if k in d})
    return p.ChunkBatch(cache=p.PagedCache(**cache), **d)


BATCH_REFUSALS = [
    ({"batch": -1}, SHAPE), ({"batch": 5}, CAPACITY), ({"total_new": -1}, SHAPE), ({"total_new": 101}, CAPACITY),
    ({"max_new_in_batch": 11}, SHAPE), ({"max_new_in_batch": -1}, SHAPE), ({"max_kv_len_in_batch": 1001}, CAPACITY),
    ({"max_kv_len_in_batch": -1}, SHAPE), ({"new_off": None}, NULL), ({"kv_len": None}, NULL), ({"k": None}, NULL),
    ({"v": None}, NULL), ({"page_table": None}, NULL), ({"n_pages": 0}, SHAPE), ({"page_size": 0}, SHAPE),
    ({"table_width": 0}, SHAPE), ({"table_stride": 4}, SHAPE), ({"page_stride": 12}, SHAPE), ({"page_stride": -64}, SHAPE),
    ({"head_stride": 4}, SHAPE), ({"row_stride": 68}, SHAPE), ({"row_stride": (1 << 24) + 8}, SHAPE),
    ({"k": FAKE + 8}, SHAPE), ({"v": FAKE + 2}, SHAPE),
]


@pytest.mark.parametrize("over,status", BATCH_REFUSALS + [({"batch": 0, "k": None}, OK), ({"total_new": 0, "max_new_in_batch": 0}, OK)])
def test_chunk_batch_refusals(p, over, status):
    st, h = _create(p, "chunk", _chunk_shape(p))
    assert st == OK
    ap = p.AppendArgs(_batch(p, **over), FAKE, FAKE, 128, 64, 128, 64)
    at = p.AttnArgs(_batch(p, **over), FAKE, 512, 64, FAKE, 512, 64, 0.0)
    assert p.lib().respec_chunk_append(h, ctypes.byref(ap), None) == status
    assert p.lib().respec_chunk_attn(h, ctypes.byref(at), FAKE, None) == status
    p.lib().respec_chunk_destroy(h)


@pytest.mark.parametrize("over,status", [
    ({"k_new": None}, NULL), ({"v_new": None}, NULL), ({"k_new": FAKE + 4}, SHAPE), ({"v_new": FAKE + 4}, SHAPE),
    ({"k_token_stride": 130}, SHAPE), ({"k_head_stride": -8}, SHAPE), ({"v_token_stride": 4}, SHAPE),
    ({"v_head_stride": 1}, SHAPE),
])
def test_append_refusals(p, over, status):
    _, h = _create(p, "chunk", _chunk_shape(p))
    d = dict(k_new=FAKE, v_new=FAKE, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64)
    d.update(over)
    a = p.AppendArgs(b=_batch(p), **d)
    assert p.lib().respec_chunk_append(h, ctypes.byref(a), None) == status
    assert p.lib().respec_chunk_append(None, ctypes.byref(a), None) == NULL
    assert p.lib().respec_chunk_append(h, None, None) == NULL
    p.lib().respec_chunk_destroy(h)


@pytest.mark.parametrize("over,status", [
    ({"q": None}, NULL), ({"out": None}, NULL), ({"q": FAKE + 8}, SHAPE), ({"out": FAKE + 8}, SHAPE),
    ({"q_token_stride": 4}, SHAPE), ({"q_head_stride": -8}, SHAPE), ({"out_token_stride": 2}, SHAPE),
    ({"out_head_stride": 68}, SHAPE), ({"scale": -1.0}, PARAM), ({"scale": float("nan")}, PARAM),
    ({"scale": float("inf")}, PARAM), ({"scale": 3e38}, PARAM),
])
def test_attn_refusals(p, over, status):
    _, h = _create(p, "chunk", _chunk_shape(p))
    d = dict(q=FAKE, q_token_stride=512, q_head_stride=64, out=FAKE, out_token_stride=512, out_head_stride=64, scale=0.0)
    d.update(over)
    a = p.AttnArgs(b=_batch(p), **d)
    f = p.lib().respec_chunk_attn
    assert f(h, ctypes.byref(a), FAKE, None) == status
    assert f(h, ctypes.byref(a), None, None) == WORKSPACE
    assert f(h, ctypes.byref(a), FAKE + 16, None) == WORKSPACE
    assert f(None, ctypes.byref(a), FAKE, None) == NULL
    assert f(h, None, FAKE, None) == NULL
    p.lib().respec_chunk_destroy(h)


@pytest.mark.parametrize("shape,status", [
    ((100, 0, 4, 8), OK), ((100, 1, 4, 16), OK), ((100, 2, 4, 8), DTYPE), ((7, 0, 4, 8), SHAPE), ((100, 0, 0, 8), SHAPE),
    ((100, 0, 4, 0), SHAPE), ((100, 0, 4, 17), SHAPE), ((1 << 30, 0, 4, 8), SHAPE), ((1, 0, 1, 1), OK),
])
def test_score_create(p, shape, status):
    st, h = _create(p, "score", p.ScoreShape(*shape))
    assert st == status
    p.lib().respec_score_destroy(h)


@pytest.mark.parametrize("over,status", [
    ({"rows": -1}, SHAPE), ({"rows": 5}, CAPACITY), ({"rows": 0, "logits": None}, OK), ({"logits": None}, NULL),
    ({"logits": FAKE + 2}, SHAPE), ({"row_stride": 99}, SHAPE),
])
def test_score_refusals(p, over, status):
    _, h = _create(p, "score", p.ScoreShape(100, 0, 4, 8))
    d = dict(rows=4, logits=FAKE, row_stride=100)
    d.update(over)
    a = p.ScoreArgs(**d)
    f = p.lib().respec_score
    assert f(h, ctypes.byref(a), FAKE, None) == status
    assert f(h, ctypes.byref(a), FAKE + 128, None) == WORKSPACE
    assert f(h, ctypes.byref(a), None, None) == WORKSPACE
    assert f(None, ctypes.byref(a), FAKE, None) == NULL
    p.lib().respec_score_destroy(h)


def test_status_string(p):
    from paper_2511_01282_amd import binding
    assert "page" in binding.status_string(p.ERR_PAGE)


def test_binding_refuses_tensors_elsewhere(p):
    """Wrong devices, types and shapes are refused before the library is called."""
    import torch
    plan = p.ChunkPlan(n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=1, max_batch=2, max_new=8, max_kv_len=64, device="cpu")
    bf, i32 = torch.bfloat16, torch.int32
    good = dict(k_new=torch.zeros(3, 2, 64, dtype=bf), v_new=torch.zeros(3, 2, 64, dtype=bf),
                k_pages=torch.zeros(5, 2, 16, 64, dtype=bf), v_pages=torch.zeros(5, 2, 16, 64, dtype=bf),
                page_table=torch.zeros(1, 4, dtype=i32), new_off=torch.zeros(2, dtype=i32), kv_len=torch.zeros(1, dtype=i32))
    for name, t in (("k_new", torch.zeros(3, 2, 64)), ("v_new", torch.zeros(3, 4, 64, dtype=bf)),
                    ("k_new", torch.zeros(3, 64, 2, dtype=bf).transpose(1, 2)),
                    ("v_pages", torch.zeros(5, 16, 2, 64, dtype=bf).transpose(1, 2)), ("new_off", torch.zeros(3, dtype=i32)),
                    ("kv_len", torch.zeros(1, dtype=torch.int64)), ("page_table", torch.zeros(2, 4, dtype=i32)),
                    ("new_off", torch.zeros(4, dtype=i32)[::2])):
        with pytest.raises(ValueError):
            plan.append(**dict(good, **{name: t}), max_new_in_batch=3)
    other = dict(good, k_new=good["k_new"].to("meta"))
    with pytest.raises(ValueError):
        plan.append(**other, max_new_in_batch=3)
    plan.close()
    with pytest.raises(ValueError):
        plan.append(**good, max_new_in_batch=3)
