"""Attention over keys of another length against its definition in 64 bits:
forward, backward, the relative position bias and its gradient, the short form."""
import ctypes
import math
import random

import pytest
import torch

import cross_reference as R
from paper_2410_11720_amd import abft

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAMES = ("O", "dQ", "dK", "dV", "dbias")


# ---- host: buckets, sizes, refusals -------------------------------------------

def test_buckets_match_whole_number_arithmetic():
    rng = random.Random(5)
    shapes = [(32, 128, True), (32, 128, False), (4, 2, True), (2, 2, False), (64, 1024, True),
              (128, 1024, True), (128, 1024, False), (8, 64, False), (10, 100, True), (7, 9, False)]
    for _ in range(60):
        two = rng.random() < 0.5
        nb = 2 * rng.randint(2, 64) if two else rng.randint(2, 128)
        e = (nb // 2 if two else nb) // 2
        shapes.append((nb, rng.randint(e + 1, 1024), two))
    for nb, top, two in shapes:
        for rel in list(range(-top - 3, top + 4)) + [-2 ** 40, 2 ** 40]:
            r = max(-2 ** 20, min(2 ** 20, rel))
            assert abft.attn_rel_bucket(rel, nb, top, two) == R.bucket(r, nb, top, two), (nb, top, two, rel)


def test_bucket_refusals():
    for nb, top, two in ((1, 128, False), (2, 128, True), (5, 128, True), (130, 128, False),
                         (32, 8, True), (32, 1025, True), (0, 128, False), (-4, 128, True)):
        with pytest.raises(abft.AbftError):
            abft.attn_rel_bucket(0, nb, top, two)


def _cfg(**kw):
    base = dict(batch=2, q_len=3, k_len=5, heads=4, head_dim=64)
    base.update(kw)
    return abft.CrossConfig(**base)


@pytest.mark.parametrize("kw", [dict(batch=-1), dict(q_len=-1), dict(k_len=-1), dict(heads=0),
                                dict(heads=4, kv_heads=3), dict(head_dim=96), dict(head_dim=0),
                                dict(scale=math.nan), dict(scale=math.inf), dict(buckets=-1),
                                dict(buckets=3), dict(buckets=32, max_distance=8),
                                dict(buckets=256), dict(q_len=2 ** 30), dict(batch=2 ** 30)])
def test_config_refusals(kw):
    with pytest.raises(abft.AbftError):
        abft.attn_cross_workspace_bytes(_cfg(**kw))


def test_workspace_bytes_cover_both_directions():
    small = abft.attn_cross_workspace_bytes(_cfg())
    assert small >= 2 * 2 * 4 * 128 * 4
    # (64 splits at most: the short form's partial results)
    assert abft.attn_cross_workspace_bytes(_cfg(k_len=8192)) <= 64 * 2 * 4 * 3 * (64 + 2) * 4 + 1024
    assert abft.attn_cross_workspace_bytes(_cfg(q_len=0, k_len=0)) > 0
    assert abft.attn_cross_workspace_bytes(_cfg(batch=0)) > 0


def _c_tensor(ptr, shape, stride=None):
    if stride is None:
        stride = (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])
    return ctypes.byref(abft.CrossTensor(ptr, *stride))


def _forward_status(cfg, q=None, k=None, o=None, bias=0, ws=1 << 20, ws_ptr=4096):
    c = cfg.to_c()
    qs = (cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
    ks = (cfg.batch, cfg.k_len, cfg.kv_heads or cfg.heads, cfg.head_dim)
    q, k = q or _c_tensor(4096, qs), k or _c_tensor(8192, ks)
    o = o or _c_tensor(4096, qs)
    return abft._lib.attn_cross_forward(c, q, k, _c_tensor(8192, ks), bias or None, None, None, o,
                                        None, None, ws_ptr, ws, None)


def test_forward_refuses_before_any_launch():
    """Pointers are never followed: the calls return first (those that pass
    every check end at the device's)."""
    cfg = _cfg()
    qs, ks = (2, 3, 4, 64), (2, 5, 4, 64)
    assert _forward_status(cfg, q=_c_tensor(4097, qs)) == -1            # alignment
    assert _forward_status(cfg, q=_c_tensor(0, qs)) == -1               # null
    assert _forward_status(cfg, q=_c_tensor(4096, qs, (768, 257, 64))) == -1
    assert _forward_status(cfg, k=_c_tensor(8192, ks, (-768, 256, 64))) == -1
    assert _forward_status(cfg, k=_c_tensor(8192, ks, (2 ** 26, 2 ** 24, 64))) == -2
    assert _forward_status(cfg, o=_c_tensor(4096, qs, (768, 0, 64))) == -1  # written twice
    assert _forward_status(cfg, o=_c_tensor(4096, qs, (768, 64, 64))) == -1  # heads on tokens
    assert _forward_status(cfg, o=_c_tensor(4096, qs, (64, 64, 768))) == -1
    assert _forward_status(cfg, bias=4096) == -1                        # a table without buckets
    assert _forward_status(_cfg(buckets=32)) == -1                      # buckets without a table
    long = _cfg(batch=1, q_len=1, k_len=8192)
    assert _forward_status(long, ws=64) == -4
    assert _forward_status(long, ws_ptr=None) == -1
    assert _forward_status(_cfg(batch=0)) == 0 and _forward_status(_cfg(q_len=0)) == 0


# ---- GPU -------------------------------------------------------------------------

def _inputs(cfg, seed, lens=None, starts=None, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[cfg.dtype]
    kvh = cfg.kv_heads or cfg.heads
    rnd = lambda *s: (torch.randn(s, generator=gen, device="cuda") * scale).to(dt)
    q = rnd(cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
    k = rnd(cfg.batch, cfg.k_len, kvh, cfg.head_dim)
    v = rnd(cfg.batch, cfg.k_len, kvh, cfg.head_dim)
    g = rnd(cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
    bias = None
    if cfg.buckets:
        bias = torch.randn((cfg.buckets, cfg.heads), generator=gen, device="cuda")
    vec = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    return q, k, v, g, dict(bias=bias, k_lens=vec(lens), q_start=vec(starts))


def _want(cfg, q, k, v, g, keys):
    return R.reference(q, k, v, g, keys["bias"], keys["k_lens"], keys["q_start"], cfg.causal,
                       cfg.scale if cfg.scale > 0 else None, cfg.max_distance, cfg.bidirectional)


def _run(cfg, q, k, v, g, keys, backward=True):
    att = abft.CrossAttention(cfg)
    att.workspace.fill_(255)       # (NaN patterns: nothing may come from there)
    o = att.forward(q, k, v, **keys)
    if not backward:
        return (o,), att
    att.workspace.fill_(255)
    return (o, *att.backward(g, q, k, v, o, **keys)), att


def _check(cfg, seed, lens=None, starts=None):
    print(f"[case] {cfg} {lens} {starts}", flush=True)
    q, k, v, g, keys = _inputs(cfg, seed, lens, starts)
    got, att = _run(cfg, q, k, v, g, keys)
    want = _want(cfg, q, k, v, g, keys)
    torch.cuda.synchronize()
    n = 5 if cfg.buckets else 4
    R.check(got[:n], want, NAMES[:n])
    R.check([att.lse], want, ["lse"])


C = abft.CrossConfig
GRID = [
    # lengths from one on, around the tiles' edges, odd ones
    (C(1, 1, 1, 1, 64), None, None),
    (C(2, 1, 77, 12, 64), [77, 40], None),
    (C(3, 33, 31, 2, 64), [31, 0, 1], None),
    (C(2, 128, 64, 2, 64), None, None),
    (C(2, 129, 65, 2, 64), [65, 64], None),
    (C(1, 127, 300, 3, 64), None, None),
    (C(2, 257, 129, 2, 128), [129, 100], None),
    (C(1, 1, 1, 1, 128), None, None),
    (C(2, 40, 200, 8, 128, kv_heads=2), [199, 3], None),
    (C(1, 70, 90, 6, 64, kv_heads=1), None, None),
    # causal: self attention, queries that start in the middle, before the
    # first key (rows without keys) and behind the last one
    (C(2, 200, 200, 2, 64, causal=True), None, None),
    (C(2, 130, 130, 4, 128, kv_heads=2, causal=True), [130, 65], None),
    (C(3, 50, 150, 2, 64, causal=True), [150, 120, 0], [100, -20, 5]),
    (C(2, 64, 40, 2, 64, causal=True), [40, 40], [1000, -63]),
    (C(2, 64, 40, 2, 64, causal=True), None, [-64, -1000000]),
    (C(2, 300, 100, 2, 128, causal=True), [100, 50], [-150, -299]),
    # bias: two-sided and one-sided, near and far, small and large tables
    (C(2, 150, 333, 3, 64, buckets=32), [333, 200], None),
    (C(2, 300, 300, 2, 64, causal=True, buckets=32, bidirectional=False), None, None),
    (C(1, 200, 260, 2, 128, buckets=32, bidirectional=False), None, None),
    (C(1, 140, 700, 2, 64, buckets=4, max_distance=2), None, None),
    (C(1, 40, 90, 2, 64, buckets=2, max_distance=2, bidirectional=False), None, None),
    (C(1, 180, 1500, 1, 64, buckets=128, max_distance=1024), None, None),
    (C(2, 90, 110, 8, 128, kv_heads=2, buckets=64, causal=True), [110, 64], [20, 0]),
    (C(2, 60, 600, 4, 64, kv_heads=2, buckets=32), [600, 0], [500, 3]),
    # full precision
    (C(1, 1, 1, 1, 64, dtype="f32"), None, None),
    (C(2, 130, 77, 2, 64, dtype="f32"), [77, 0], None),
    (C(2, 65, 140, 4, 128, kv_heads=2, dtype="f32"), [140, 33], None),
    (C(2, 150, 150, 2, 64, dtype="f32", causal=True, buckets=32, bidirectional=False), None, None),
    (C(1, 100, 300, 2, 128, dtype="f32", buckets=32), None, None),
    # few heads over long axes (waves that share queries or keys), many heads
    (C(1, 330, 700, 2, 64, buckets=32), [650], None),
    (C(1, 500, 500, 4, 128, causal=True, buckets=32, bidirectional=False), None, None),
    (C(2, 260, 300, 2, 128, kv_heads=1), [300, 40], None),
    (C(2, 250, 340, 2, 64, dtype="f32", causal=True), [340, 100], [90, -30]),
    (C(1, 130, 500, 4, 128, dtype="f32", buckets=32), None, None),
    (C(4, 64, 90, 100, 64, buckets=32), [90, 64, 33, 0], None),
    (C(3, 70, 150, 60, 128, causal=True, buckets=32), [150, 129, 2], [80, 59, 0]),
    (C(4, 45, 40, 90, 64, dtype="f32"), [40, 33, 32, 1], None),
    (C(1, 96, 800, 2, 128, buckets=128, max_distance=1024), None, None),
    (C(1, 96, 800, 2, 128, dtype="f32", buckets=128, max_distance=1024), None, None),
    (C(1, 96, 800, 2, 64, dtype="f32", buckets=128, max_distance=1024), None, None),
    # one axis over several workgroups, whose sums are joined
    (C(1, 600, 40, 8, 64, kv_heads=1, buckets=32), [37], None),
    (C(2, 525, 25, 8, 64, kv_heads=1, dtype="f32"), [25, 0], None),
    (C(1, 40, 2000, 1, 128), [1990], None),
    (C(2, 33, 1500, 2, 64, buckets=32), [1500, 70], [700, -5]),
    (C(1, 700, 700, 2, 64, causal=True, buckets=32, bidirectional=False), None, None),
    (C(2, 300, 900, 4, 128, kv_heads=1, causal=True, buckets=8), [900, 31], [600, -270]),
    (C(1, 90, 1100, 2, 128, dtype="f32", buckets=32), None, None),
    (C(1, 800, 90, 6, 128, kv_heads=2, dtype="f32", causal=True), None, [-100]),
    # another scale
    (C(1, 50, 60, 2, 64, scale=0.3), None, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(GRID)))
def test_forward_and_backward(n):
    cfg, lens, starts = GRID[n]
    _check(cfg, 100 + n, lens, starts)


# decoded tokens: splits over a long cache, several tiles of shared rows
SHORT = [
    (C(1, 1, 5000, 1, 64), None, None),
    (C(2, 1, 4097, 4, 128, kv_heads=1), [4097, 4096], None),
    (C(3, 4, 3000, 20, 128, kv_heads=2, causal=True), [3000, 1, 0], [2996, -3, -4]),
    (C(2, 32, 1000, 4, 64, kv_heads=2, causal=True), [1000, 500], [968, 468]),
    (C(4, 1, 2500, 12, 64, causal=True, buckets=32, bidirectional=False), [2500, 129, 128, 1],
     [2499, 128, 127, 0]),
    (C(2, 3, 700, 64, 64, kv_heads=1, buckets=128, max_distance=1024), [700, 650], [350, 0]),
    (C(2, 2, 900, 2, 128, dtype="f32", buckets=32), [900, 10], [450, 10]),
    (C(2, 1, 2100, 4, 64, dtype="f32", kv_heads=2), [2100, 0], None),
    (C(70, 1, 40, 12, 64), [1 + (7 * i) % 40 for i in range(70)], None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(SHORT)))
def test_short_form(n):
    cfg, lens, starts = SHORT[n]
    _check(cfg, 200 + n, lens, starts)


# more workgroups of the query pass than the chip holds two a CU: of 64 and of
# 128 queries
_LENS = [130 - 11 * (i % 5) if i % 7 else 0 for i in range(16)]
MANY = [
    (C(16, 140, 200, 16, 64), None, None),
    (C(16, 140, 130, 16, 64, causal=True, buckets=32), _LENS, [n - 140 for n in _LENS]),
    (C(16, 300, 130, 16, 64), _LENS, None),
    (C(16, 300, 130, 16, 64, kv_heads=4, causal=True, buckets=32, bidirectional=False), None, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(MANY)))
def test_many_workgroups(n):
    cfg, lens, starts = MANY[n]
    _check(cfg, 300 + n, lens, starts)


# fp32, few keys (queries): waves that share 32 rows have one block of the other
# axis each, or a part of one, or none
FEW = [C(3, q, k, 2, d, dtype="f32", causal=causal, buckets=buckets)
       for q, k, d, causal, buckets in [(61, 47, 128, False, 0), (33, 33, 128, True, 32),
                                        (100, 97, 64, False, 32), (97, 128, 64, True, 0),
                                        (128, 33, 64, False, 0), (40, 200, 128, False, 32)]]


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [None, [1, 1000, 0], [32, 31, 33]])
@pytest.mark.parametrize("n", range(len(FEW)))
def test_few_blocks(n, lens):
    cfg = FEW[n]
    _check(cfg, 400 + n, lens and [min(x, cfg.k_len) for x in lens], None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,q_len", [("bf16", 64, 70), ("bf16", 128, 2), ("f32", 64, 70),
                                           ("f32", 128, 1)])
def test_views_of_packed_and_transposed_tensors(dtype, d, q_len):
    """Queries from a packed tensor, keys from a [batch, heads, tokens] cache
    larger than its use, values the same for all sequences, outputs into views:
    what lies around them stays."""
    cfg = C(2, q_len, 90, 4, d, kv_heads=2, dtype=dtype, buckets=32)
    gen = torch.Generator(device="cuda").manual_seed(9)
    dt = DT[dtype]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    packed = rnd(2, q_len, 4, 3, d)
    q, g = packed[:, :, :, 1], rnd(4, q_len, 2, d).transpose(0, 2)
    cache = rnd(2, 2, 130, d)
    k = cache[:, :, 17:107].transpose(1, 2)
    v = rnd(90, 2, d).unsqueeze(0).expand(2, -1, -1, -1)
    keys = dict(bias=rnd(32, 4).float(), k_lens=torch.tensor([90, 61], dtype=torch.int32,
                                                              device="cuda"), q_start=None)
    assert not (q.is_contiguous() or k.is_contiguous() or g.is_contiguous())
    att = abft.CrossAttention(cfg)
    box = torch.full((2, q_len + 3, 6, d + 8 * 16 // dt.itemsize), 7.0, dtype=dt, device="cuda")
    o = box[:, 1:q_len + 1, 1:5, :d]
    kbox = torch.full((2, 2, 2, 95, d), 7.0, dtype=dt, device="cuda")
    dk, dv = kbox[0, :, :, 2:92].transpose(1, 2), kbox[1, :, :, 2:92].transpose(1, 2)
    att.forward(q, k, v, O=o, **keys)
    got = (o, *att.backward(g, q, k, v, o, dK=dk, dV=dv, **keys))
    R.check(got, _want(cfg, q, k, v, g, keys), NAMES)
    o.fill_(7.0)
    dk.fill_(7.0)
    dv.fill_(7.0)
    assert (box == 7).all() and (kbox == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,q_len", [("bf16", 65), ("bf16", 1), ("f32", 65), ("f32", 1)])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -3e38])
def test_what_lies_behind_a_sequence_is_not_used(dtype, q_len, junk):
    cfg = C(3, q_len, 200, 2, 64, dtype=dtype, buckets=32)
    lens = [200, 67, 0]
    q, k, v, g, keys = _inputs(cfg, 31, lens)
    clean, att = _run(cfg, q, k, v, g, keys)
    lse = att.lse.clone()
    for b, n in enumerate(lens):
        k[b, n:] = junk
        v[b, n:] = junk
    dirty, att = _run(cfg, q, k, v, g, keys)
    for a, b in zip(clean, dirty):
        assert torch.equal(a, b)
    assert torch.equal(lse, att.lse)
    o, dq, dk, dv, _ = dirty
    assert (o[2] == 0).all() and (dq[2] == 0).all() and (att.lse[2] == -math.inf).all()
    for b, n in enumerate(lens):
        assert (dk[b, n:] == 0).all() and (dv[b, n:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, -2e30, -math.inf])
@pytest.mark.parametrize("q_len", [70, 3])
def test_bias_of_the_types_lowest_value_masks(low, q_len):
    """A table entry below -1e30 takes its bucket's keys out, near and far,
    also where that leaves a row without keys."""
    cfg = C(1, q_len, 300, 1, 64, buckets=4, max_distance=2)
    q, k, v, g, keys = _inputs(cfg, 5)
    keys["bias"][2:, :] = low              # keys ahead
    got, att = _run(cfg, q, k, v, g, keys)
    causal = C(1, q_len, 300, 1, 64, causal=True, buckets=4, max_distance=2)
    finite = dict(keys, bias=keys["bias"].clone())
    finite["bias"][2:, :] = 0.0
    R.check(got[:4], _want(causal, q, k, v, g, finite), NAMES[:4])
    assert (got[4][2:] == 0).all()
    keys["bias"][:] = low
    got, att = _run(cfg, q, k, v, g, keys)
    assert all((t == 0).all() for t in got) and (att.lse == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of some hundreds: the running maximum moves far and often."""
    cfg = C(1, 70, 500, 2, 64, dtype=dtype)
    q, k, v, g, keys = _inputs(cfg, 77)
    k = (k * torch.linspace(0.1, 40, 500, device="cuda")[None, :, None, None]).to(k.dtype)
    got, att = _run(cfg, q, k, v, g, keys)
    R.check(got[:4], _want(cfg, q, k, v, g, keys), NAMES[:4])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(0, 5, 5), (2, 0, 5), (2, 5, 0), (2, 0, 0)])
def test_no_elements(shape):
    B, Sq, Sk = shape
    for buckets in (0, 32):
        cfg = C(B, Sq, Sk, 2, 64, buckets=buckets)
        q, k, v, g, keys = _inputs(cfg, 3)
        got, att = _run(cfg, q, k, v, g, keys)
        for t in got:
            assert t is None or (t == 0).all()


@pytest.mark.gpu
def test_gradients_against_differences():
    """In full precision: the loss sum(w O) along a random direction of every
    input, by central differences of the forward in fp32: the step h = 2^-6 leaves a
    third-order term of about h^2 and a rounding of about 2^-24 sqrt(n) / h of
    the loss's magnitude."""
    cfg = C(2, 20, 33, 2, 64, dtype="f32", buckets=32)
    q, k, v, g, keys = _inputs(cfg, 8, [33, 17])
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v, **keys)
    grads = att.backward(g, q, k, v, o, **keys)
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = 2.0 ** -6
    for at in range(4):
        x = (q, k, v, keys["bias"])[at]
        step = torch.randn(x.shape, generator=gen, device="cuda")
        step /= step.norm()
        ends = []
        for s in (h, -h):
            args = [q, k, v, keys["bias"]]
            args[at] = x + s * step
            o2 = att.forward(*args[:3], bias=args[3], k_lens=keys["k_lens"])
            ends.append((o2.double() * g.double()).sum())
        num = (ends[0] - ends[1]) / (2 * h)
        ana = (grads[at].double() * step.double()).sum()
        size = (o.double() * g.double()).abs().sum()
        tol = 4 * h * h * abs(ana).item() + 2 ** -24 / h * size.item() + 1e-3 * h
        assert abs(num - ana) <= tol, (at, num.item(), ana.item(), tol)


@pytest.mark.gpu
def test_runs_repeat_bit_for_bit_on_any_stream():
    cfg = C(2, 150, 400, 4, 64, kv_heads=2, buckets=32)
    q, k, v, g, keys = _inputs(cfg, 12, [400, 300])
    first, att = _run(cfg, q, k, v, g, keys)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second, att2 = _run(cfg, q, k, v, g, keys)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 130])
def test_captured_calls_replay(q_len):
    """Two captured layers that share a workspace in turn, replayed with new
    inputs between eager calls."""
    cfg = C(2, q_len, 1500, 4, 64, buckets=32)
    q, k, v, g, keys = _inputs(cfg, 12, [1500, 700])
    att = abft.CrossAttention(cfg)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    grads = [torch.empty_like(t) for t in (q, k, v, keys["bias"])]

    def both():
        att.forward(q, k, v, O=o, **keys)
        att.forward(o, k, v, O=o2, **keys)
        att.backward(g, o, k, v, o2, dQ=grads[0], dK=grads[1], dV=grads[2], dbias=grads[3], **keys)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (21, 22, 23):
        fresh = _inputs(cfg, seed)[:4]
        for t, f in zip((q, k, v, g), fresh):
            t.copy_(f)
        both()
        want = [t.clone() for t in (o, o2, *grads)]
        for t in (o, o2, *grads):
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((o, o2, *grads), want):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache whose last sequence starts past 2^32 bytes, and tokens whose
    rows are 1 MiB apart."""
    cap, heads, d = 17000, 16, 128
    cache = torch.empty((2, 2, cap, heads, d), dtype=torch.bfloat16, device="cuda").normal_()
    far = torch.empty((4200, 8, 512, d), dtype=torch.bfloat16, device="cuda")   # 4.4 GB
    far[:, 0, 0].normal_()
    far[:, 1, 0].normal_()
    cfg = C(1, 2, 4200, 1, d)
    k, v = far[:, 0, :1].unsqueeze(0), far[:, 1, :1].unsqueeze(0)
    q = torch.randn((1, 2, 1, d), device="cuda").bfloat16()
    att = abft.CrossAttention(cfg)
    want = R.reference(q, k, v)
    R.check([att.forward(q, k, v)], want, ["O"])
    cfg = C(1, 160, 4200, 1, d)
    q = torch.randn((1, 160, 1, d), device="cuda").bfloat16()
    g = torch.randn((1, 160, 1, d), device="cuda").bfloat16()
    got, att = _run(cfg, q, k, v, g, {})
    R.check(got[:4], R.reference(q, k, v, g), NAMES[:4])


@pytest.mark.gpu
def test_python_refusals():
    cfg = C(2, 3, 5, 4, 64, buckets=32)
    q, k, v, g, keys = _inputs(cfg, 1)
    att = abft.CrossAttention(cfg)
    bad = [(q.float(), k, v, keys), (q, k[:, :4], v, keys), (q.cpu(), k, v, keys),
           (q, k, v, dict(keys, bias=None)), (q, k, v, dict(keys, bias=keys["bias"].bfloat16())),
           (q, k, v, dict(keys, k_lens=torch.tensor([5, 5], device="cuda"))),
           (q, k, v, dict(keys, k_lens=torch.tensor([5], dtype=torch.int32, device="cuda"))),
           (q, k, v, dict(keys, q_start=torch.tensor([0, 0], dtype=torch.int32))),
           (q.transpose(2, 3).contiguous().transpose(2, 3), k, v, keys)]
    for a, b, c, kw in bad:
        with pytest.raises(abft.AbftError):
            att.forward(a, b, c, **kw)
    with pytest.raises(abft.AbftError):
        att.backward(g, q, k, v, q[:, :2], **keys)
