"""Relative position bias whose entries are far from 0 but not masks (-1e6,
-1e9): next to such an entry a score of ordinary size, or the logarithm of a
row's sum, has few or no bits left in fp32. Rows of such keys alone keep weights
that sum to one, forward and backward."""
import pytest
import torch

import cross_reference as R
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


# far: every pair but the diagonal's lies in a constant side; near: none does.
# Tiled and short forms, waves and workgroups that share an axis, shared heads
FAR, NEAR = dict(buckets=4, max_distance=2), dict(buckets=128, max_distance=1024)
SHAPES = [dict(batch=2, q_len=70, k_len=300, heads=2, head_dim=64),
          dict(batch=1, q_len=40, k_len=1000, heads=2, head_dim=128),
          dict(batch=16, q_len=300, k_len=130, heads=16, head_dim=64),
          dict(batch=1, q_len=5, k_len=900, heads=8, head_dim=64, kv_heads=2),
          dict(batch=1, q_len=300, k_len=25, heads=8, head_dim=128, kv_heads=1),
          dict(batch=2, q_len=64, k_len=90, heads=2, head_dim=64, dtype="f32"),
          dict(batch=1, q_len=33, k_len=700, heads=2, head_dim=128, dtype="f32"),
          dict(batch=4, q_len=3, k_len=40, heads=4, head_dim=64, dtype="f32")]


@pytest.mark.gpu
@pytest.mark.parametrize("side", ["far", "near"])
@pytest.mark.parametrize("entry", [-1e4, -1e6, -1e9, 3e8, -1e29])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_weights_sum_to_one(n, entry, side):
    """With P a row's weights: sum_j dv_j = sum_i dO_i (sum_j P_ij = 1) and
    sum_t dbias_t = 0. In the first each P is off by the storage type's half
    step u and each dv too, the row's factor and the sums by fewer than 2^6
    roundings of fp32 beside n of the sum itself. The second: dS of a pair is off
    by P times (the row's largest |dP - D|) times the same, dP and D by d + 4
    roundings of at most |dO| . |v|."""
    cfg = C(**SHAPES[n], **(FAR if side == "far" else NEAR))
    print(f"[case] {cfg} {entry}", flush=True)
    q, k, v, g = _inputs(cfg, 300 + n)
    g = g.abs()
    table = torch.full((cfg.buckets, cfg.heads), entry, device="cuda")
    o, dq, dk, dv, db = _run(cfg, q, k, v, g, bias=table)
    assert all(t.isfinite().all() for t in (o, dq, dk, dv, db))
    assert (o.double().abs().amax(1) <= 1.01 * v.double().abs().amax(1).repeat_interleave(
        cfg.heads // v.shape[2], 1)).all()
    u, v32 = torch.finfo(q.dtype).eps / 2, 2.0 ** -24
    kvh = v.shape[2]
    want = g.double().sum(1).view(cfg.batch, kvh, -1, cfg.head_dim).sum(2)
    many = 64 + cfg.q_len * (cfg.heads // kvh) + cfg.k_len
    assert ((dv.double().sum(1) - want).abs() <= (2 * u + many * v32) * want).all()
    most = (g.double().abs().sum(3) * v.double().abs().amax((1, 3)).repeat_interleave(
        cfg.heads // kvh, 1)[:, None]).sum((0, 1))      # of each head: sum of |dO| . max |v|
    off = db.double().sum(0).abs()
    assert (off <= (cfg.head_dim + 4 + many) * v32 * 4 * most).all()


@pytest.mark.gpu
@pytest.mark.parametrize("zero", ["Q", "K"])
@pytest.mark.parametrize("side", ["far", "near"])
@pytest.mark.parametrize("entry", [-1e6, -1e9, -1e29])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_one_entry_for_all_pairs_changes_nothing(n, entry, side, zero):
    """Equal scores: every sum with the entry is the same number, so the results
    are those of a table of zeros, within the same bounds."""
    cfg = C(**SHAPES[n], **(FAR if side == "far" else NEAR))
    print(f"[case] {cfg} {entry} {zero}", flush=True)
    q, k, v, g = _inputs(cfg, 400 + n)
    (q if zero == "Q" else k).zero_()
    table = torch.full((cfg.buckets, cfg.heads), entry, device="cuda")
    got = _run(cfg, q, k, v, g, bias=table)
    want = R.reference(q, k, v, g, torch.zeros_like(table), None, None, False, None,
                       cfg.max_distance, True)
    R.check(got, want, ("O", "dQ", "dK", "dV", "dbias"))


@pytest.mark.gpu
@pytest.mark.parametrize("entry", [-1e6, -1e9])
@pytest.mark.parametrize("n", range(len(SHAPES)))
def test_rows_that_see_large_entries_beside_rows_that_do_not(n, entry):
    """Zero for keys behind the query and the nearest ones, the entry for those
    far ahead; the first queries lie far in front of every key. With equal scores
    the results are those of any entry that leaves no weight beside 0: of -200
    (2^-288 in weight)."""
    cfg = C(**SHAPES[n], buckets=8, max_distance=20)
    q, k, v, g = _inputs(cfg, 500 + n)
    q.zero_()
    start = torch.full((cfg.batch,), -cfg.q_len // 2 - 20, dtype=torch.int32, device="cuda")
    table = torch.zeros((8, cfg.heads), device="cuda")
    table[7] = entry
    got = _run(cfg, q, k, v, g, bias=table, q_start=start)
    table[7] = -200.0
    want = R.reference(q, k, v, g, table, None, start, False, None, 20, True)
    R.check(got, want, ("O", "dQ", "dK", "dV", "dbias"))


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
