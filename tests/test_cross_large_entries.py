"""Relative position bias whose entries are far from 0 but not masks (-1e6,
-1e9): next to such an entry a score of ordinary size, or the logarithm of a
row's sum, has few or no bits left in fp32. Rows of such keys alone keep weights
that sum to one, forward and backward."""
import pytest
import torch

from paper_2410_11720_amd import abft

C = abft.CrossConfig
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(cfg, seed, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    kvh = cfg.kv_heads or cfg.heads
    q, g = (rnd(cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim) for _ in range(2))
    k, v = (rnd(cfg.batch, cfg.k_len, kvh, cfg.head_dim) for _ in range(2))
    return [t.to(DT[cfg.dtype]) for t in (q * size, k, v, g)]


def _run(cfg, q, k, v, g, **keys):
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v, **keys)
    att.workspace.fill_(255)       # (NaN patterns: nothing may come from there)
    return (o, *att.backward(g, q, k, v, o, **keys))


# every pair but the diagonal's lies in a constant side; none does
FAR, NEAR = dict(buckets=4, max_distance=2), dict(buckets=128, max_distance=1024)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,q_len", [("bf16", 64, 70), ("bf16", 128, 2), ("f32", 64, 300),
                                           ("f32", 128, 1)])
@pytest.mark.parametrize("entry", [-1e10, -1e20, 1e10])
def test_large_scores_on_large_entries(dtype, d, q_len, entry):
    """Scores of some hundreds beside an entry that takes all their bits: finite
    results, inside the values' range (of which the output's rounding takes it by
    a step of the type at most)."""
    cfg = C(1, q_len, 600, 2, d, dtype=dtype, **FAR)
    q, k, v, g = _inputs(cfg, 7, 200.0)
    table = torch.full((4, 2), entry, device="cuda")
    out = _run(cfg, q, k, v, g, bias=table)
    assert all(t.isfinite().all() for t in out)
    lo, hi = v.double().amin(1, keepdim=True), v.double().amax(1, keepdim=True)
    wide = 2 * torch.finfo(q.dtype).eps * torch.maximum(lo.abs(), hi.abs()) + 600 * 2.0 ** -24
    assert ((out[0] >= lo - wide) & (out[0] <= hi + wide)).all()
