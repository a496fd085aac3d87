"""Attention over keys of another length with values that are not finite:
what a query sees reaches its results, what it does not see stays out of them."""
import math

import pytest
import torch

from paper_2410_11720_amd import abft

C = abft.CrossConfig
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(cfg, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DT[cfg.dtype])
    kvh = cfg.kv_heads or cfg.heads
    q, g = (rnd(cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim) for _ in range(2))
    k, v = (rnd(cfg.batch, cfg.k_len, kvh, cfg.head_dim) for _ in range(2))
    return q, k, v, g


# each way to spread a forward over waves and workgroups: four waves on the
# queries, two, one; decoded tokens in one piece and over several workgroups
FORMS = [C(8, 600, 300, 32, 64, causal=True), C(2, 150, 300, 2, 128, causal=True),
         C(1, 64, 200, 2, 64, causal=True), C(1, 64, 200, 2, 64, dtype="f32", causal=True),
         C(1, 130, 300, 2, 128, dtype="f32", causal=True), C(2, 8, 200, 4, 64, causal=True),
         C(1, 4, 3000, 8, 128, kv_heads=2, causal=True),
         C(1, 4, 3000, 2, 128, dtype="f32", causal=True)]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(FORMS)))
@pytest.mark.parametrize("back", [1, 33, 70])
def test_a_nan_key_reaches_the_queries_that_see_it(n, back):
    """The queries are the last positions; key `at` holds NaN: rows in front of
    it as without it, rows from it on NaN, O and lse."""
    cfg = FORMS[n]
    print(f"[case] {cfg} {back}", flush=True)
    q, k, v, _ = _inputs(cfg, 60 + n)
    begin = max(0, cfg.k_len - cfg.q_len)
    at = max(0, cfg.k_len - back)
    start = torch.full((cfg.batch,), begin, dtype=torch.int32, device="cuda")
    att = abft.CrossAttention(cfg)
    clean = att.forward(q, k, v, q_start=start)
    lse = att.lse.clone()
    k[:, at] = math.nan
    o = att.forward(q, k, v, q_start=start)
    first = max(0, at - begin)
    assert torch.equal(o[:, :first], clean[:, :first])
    assert torch.equal(att.lse[:, :, :first], lse[:, :, :first])
    assert o[:, first:].isnan().all() and att.lse[:, :, first:].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("k_len", [64, 256])
def test_queries_that_see_nothing_but_nan(dtype, d, k_len):
    """A table that leaves each query the key at its own position, and NaN in
    the last 32 keys: the wave that holds them finds no maximum, the others no
    key at all."""
    cfg = C(1, 40, k_len, 1, d, dtype=dtype, buckets=4, max_distance=2)
    q, k, v, g = _inputs(cfg, 5)
    table = torch.tensor([[0.0], [-math.inf], [0.0], [-math.inf]], device="cuda")
    start = torch.tensor([k_len - 32], dtype=torch.int32, device="cuda")
    k[:, k_len - 32:] = math.nan
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v, bias=table, q_start=start)
    assert o[:, :32].isnan().all() and att.lse[:, :, :32].isnan().all()
    dq, _, dv, _ = att.backward(g, q, k, v, o, bias=table, q_start=start)
    assert dq[:, :32].isnan().all() and dv[:, k_len - 32:].isnan().all()


# queries in front of the first key; a query pass of one, two, four waves on
# the queries, its other axis over several workgroups; a key pass likewise
AHEAD = [C(2, 90, 60, 2, 64, causal=True), C(8, 300, 200, 32, 64, causal=True),
         C(2, 200, 300, 4, 128, kv_heads=2, causal=True), C(1, 700, 64, 2, 64, causal=True),
         C(1, 80, 1500, 1, 128, causal=True), C(2, 90, 60, 2, 64, dtype="f32", causal=True),
         C(1, 300, 90, 2, 128, dtype="f32", causal=True),
         C(2, 150, 150, 2, 64, causal=True, buckets=32)]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(AHEAD)))
@pytest.mark.parametrize("ahead", [1, 37, 64])
@pytest.mark.parametrize("junk", [math.nan, math.inf])
def test_no_gradient_comes_from_a_query_without_keys(n, ahead, junk):
    """Whatever Q and dO hold there (padding in front of a sequence)."""
    cfg = AHEAD[n]
    print(f"[case] {cfg} {ahead} {junk}", flush=True)
    q, k, v, g = _inputs(cfg, 80 + n)
    keys = dict(q_start=torch.full((cfg.batch,), -ahead, dtype=torch.int32, device="cuda"))
    if cfg.buckets:
        keys["bias"] = torch.randn((cfg.buckets, cfg.heads), device="cuda")
    att = abft.CrossAttention(cfg)
    results = []
    for fill in (0.0, junk):
        q[:, :ahead] = fill
        g[:, :ahead] = fill
        o = att.forward(q, k, v, **keys)
        results.append((o, *att.backward(g, q, k, v, o, **keys)))
    for a, b in zip(*results):
        assert a is None or torch.equal(a, b)
    o, dq = results[1][:2]
    assert (o[:, :ahead] == 0).all() and (dq[:, :ahead] == 0).all()
    assert (att.lse[:, :, :ahead] == -math.inf).all()
