"""Entropies of verification steps whose logits are very low for most of the vocabulary.

The residual's first column is 1 and a masked word's LM-head row is the low value there, so its logit is that value
exactly.  The statistics are compared with those of the returned logits in 64 bits: log-sum-exp to 1e-5 and a rounding,
entropy to 1.2e-4, as in test_gpu_lmhead_tiles.py (both bounds are derived there)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low", [-3.3e38, -1e38, -1e37, -1e20])
@pytest.mark.parametrize("dtype,m,hidden,vocab", [
    ("f32", 1, 128, 4099), ("f32", 19, 128, 32000), ("bf16", 1, 256, 16449), ("bf16", 26, 256, 32000), ("bf16", 33, 512, 20001),
    ("bf16", 65, 256, 32001), ("bf16", 257, 256, 32004), ("bf16", 40, 256, 150001),
])
def test_entropy_beside_low_logits(dtype, m, hidden, vocab, low):
    from paper_2511_01282_amd import binding
    dev, dt = "cuda:0", torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator(device=dev).manual_seed(m)
    heads, batch = hidden // 64, -(-m // 64)
    nodes = [m // batch + (1 if b < m % batch else 0) for b in range(batch)]

    def rand(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device=dev) * std).to(dt)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    h, w = rand(m, hidden), rand(vocab, hidden, std=0.1)
    h[:, 0], w[:, 0] = 1.0, 0.0
    ids = torch.arange(vocab, device=dev)
    keep = (ids % 4096 == 70) | ((ids > 1000) & (ids < 1200))
    w[~keep] = 0.0
    w[~keep, 0] = low
    ins = dict(node_off=ints([sum(nodes[:b]) for b in range(batch + 1)]), kv_len=ints([0] * batch), hidden=h,
               k_cache=rand(batch, heads, 64, 64), v_cache=torch.zeros(batch, heads, 64, 64, dtype=dt, device=dev), lm_head=w,
               parent=ints([j - 1 for n in nodes for j in range(n)]), token=ints([1001] * m),
               src=torch.zeros(m, dtype=torch.uint8, device=dev))
    plan = binding.Plan(hidden=hidden, n_q_heads=heads, n_kv_heads=heads, head_dim=64, vocab=vocab,
                        dtype=binding.F32 if dtype == "f32" else binding.BF16, max_batch=batch, max_nodes=64, max_depth=64,
                        max_kv_len=0, topk_out=8)
    out = binding.alloc_outputs(total_nodes=m, batch=batch, hidden=hidden, vocab=vocab, topk_out=8, max_depth=64)
    plan.step(ins, out, batch=batch, total_nodes=m, max_nodes_in_batch=max(nodes), max_kv_len_in_batch=0,
              kv_capacity=64, topk=8, stop_after=binding.STOP_STATS)
    torch.cuda.synchronize()
    z = out["logits"].double()
    assert bool(z.isfinite().all()) and bool((z[:, ~keep] == torch.tensor(low, dtype=dt).double().item()).all())
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    assert float((out["lse"] - lse).abs().max()) <= 1e-5 + 2.0 ** -23 * float(lse.abs().max())
    assert float((out["entropy"] - entropy).abs().max()) <= 1.2e-4
    assert bool(out["entropy"].isfinite().all())
