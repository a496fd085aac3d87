"""Rotary positions against their definition in 64 bits: both layouts of pairs,
parts of a head, far positions, the backward, the append to a cache; refusals."""
import ctypes
import math

import pytest
import torch

import block_reference as R
from paper_2410_11720_amd import abft

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
C = abft.RotaryConfig


# ---- host ------------------------------------------------------------------------------

def test_frequencies():
    f = abft.attn_rotary_frequencies
    for n, base in ((2, 10000.0), (64, 10000.0), (128, 5e5), (20, 2.0)):
        want = [math.exp(-2 * k / n * math.log(base)) for k in range(n // 2)]
        assert f(n, base) == pytest.approx(want, rel=1e-14)
        assert f(n, base, "linear", 4.0) == pytest.approx([w / 4 for w in want], rel=1e-14)
        parts = f(n, base, "parts", 8.0, 4096, 2.0, 16.0)
        for w, p in zip(want, parts):
            turns = 4096 * w / (2 * math.pi)
            keep = min(1, max(0, (turns - 2) / 14))
            assert p == pytest.approx(w * (keep + (1 - keep) / 8), rel=1e-14)
            assert w / 8 * (1 - 1e-14) <= p <= w * (1 + 1e-14)
    assert f(0) == []


def test_frequency_refusals():
    f = abft.attn_rotary_frequencies
    for args in ((3,), (-2,), (1024,), (8, 0.0), (8, math.nan), (8, math.inf),
                 (8, 1e4, "linear", 0.0), (8, 1e4, "linear", math.inf), (8, 1e4, "other"),
                 (8, 1e4, "parts", 2.0, 0.0), (8, 1e4, "parts", 2.0, 2048, 4.0, 4.0),
                 (8, 1e4, "parts", 2.0, 2048, -1.0, 4.0), (8, 1e4, "parts", math.nan)):
        with pytest.raises(abft.AbftError):
            f(*args)


G = 1 << 30
ST = (192, 64, 16)          # [2, 3, 4, 16]


def _t(ptr, stride=ST):
    return ctypes.byref(abft.CrossTensor(ptr, *stride))


def _status(q=None, k=None, qo=None, ko=None, freqs=7 * G, start=None, backward=0, **kw):
    base = dict(batch=2, tokens=3, heads=4, head_dim=16)
    base.update(kw)
    return abft._lib.attn_rotary(C(**base).to_c(), backward, q or _t(G), k or _t(2 * G), freqs, start,
                                 qo or _t(3 * G), ko or _t(4 * G), None)


def _append(q=None, k=None, v=None, qo=None, kc=None, vc=None, freqs=7 * G, start=None, capacity=9,
            **kw):
    base = dict(batch=2, tokens=3, heads=4, head_dim=16)
    base.update(kw)
    cs = (9 * 64, 64, 16)
    return abft._lib.attn_rotary_append(C(**base).to_c(), q or _t(G), k or _t(2 * G), v or _t(3 * G),
                                        freqs, start, capacity, qo or _t(4 * G), kc or _t(5 * G, cs),
                                        vc or _t(6 * G, cs), None)


def test_refusals_before_any_launch():
    """Pointers are never followed: the calls return first."""
    for kw in (dict(batch=-1), dict(tokens=-1), dict(heads=-1), dict(head_dim=0), dict(kv_heads=-1),
               dict(rotary_dim=3), dict(rotary_dim=18), dict(rotary_dim=-2), dict(head_dim=15),
               dict(magnitude=math.nan), dict(magnitude=math.inf), dict(backward=2), dict(freqs=None),
               dict(freqs=7 * G + 4), dict(start=8 * G + 2)):
        assert _status(**kw) == -1, kw
    for kw in (dict(head_dim=514), dict(heads=65536, kv_heads=1), dict(batch=2 ** 16, tokens=2 ** 15)):
        assert _status(**kw) == -2, kw
    assert _status(q=_t(0)) == -1 and _status(ko=_t(0)) == -1 and _status(k=_t(2 * G + 1)) == -1
    assert _status(q=_t(G, (192, -64, 16))) == -1 and _status(qo=_t(3 * G, (192, 0, 16))) == -1
    assert _status(qo=_t(3 * G, (192, 64, 15))) == -1
    # in place is each on its own, exactly
    assert _status(qo=_t(G + 2)) == -1 and _status(qo=_t(2 * G)) == -1 and _status(ko=_t(G)) == -1
    assert _status(ko=_t(3 * G)) == -1 and _status(qo=_t(7 * G)) == -1
    assert _status(qo=_t(G, (64, 128, 16))) == -1
    assert _status(start=3 * G) == -1
    assert _status(batch=0) == 0 and _status(tokens=0, q=_t(0)) == 0
    assert _append(capacity=-1) == -1
    assert _append(kc=_t(6 * G, (576, 64, 16))) == -1 and _append(vc=_t(5 * G + 64, (576, 64, 16))) == -1
    assert _append(kc=_t(2 * G)) == -1 and _append(vc=_t(G, (576, 64, 16))) == -1
    assert _append(kc=_t(5 * G, (64, 64, 16))) == -1 and _append(v=_t(0)) == -1
    assert _append(qo=_t(2 * G)) == -1 and _append(qo=_t(3 * G)) == -1
    assert _append(batch=0) == 0


def test_python_refusals_without_a_gpu():
    rot = abft.Rotary(C(2, 3, 4, 16, kv_heads=2), device="cpu")
    q, k = torch.zeros((2, 3, 4, 16)).bfloat16(), torch.zeros((2, 3, 2, 16)).bfloat16()
    for args in ((q, q), (q.float(), k), (q[:, :2], k), (q.transpose(2, 3), k)):
        with pytest.raises(abft.AbftError):
            rot.forward(*args)
    with pytest.raises(abft.AbftError):
        rot.forward(q, k, q_start=torch.zeros(2))
    with pytest.raises(abft.AbftError):
        rot.append(q, k, k, torch.zeros((2, 9, 2, 16)), torch.zeros((2, 9, 2, 16)))
    for kw in (dict(scaling="other"), dict(rotary_dim=7), dict(dtype="f16")):
        with pytest.raises(abft.AbftError):
            abft.Rotary(C(2, 3, 4, 16, **kw), device="cpu")


# ---- GPU -------------------------------------------------------------------------------

def _inputs(cfg, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kvh = cfg.kv_heads or cfg.heads
    rnd = lambda h: torch.randn((cfg.batch, cfg.tokens, h, cfg.head_dim), generator=gen,
                                device="cuda").to(DT[cfg.dtype])
    return rnd(cfg.heads), rnd(kvh), rnd(kvh)


def _start(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def _check(cfg, seed, starts=None):
    print(f"[case] {cfg} {starts}", flush=True)
    q, k, _ = _inputs(cfg, seed)
    rot = abft.Rotary(cfg)
    at = starts or [0] * cfg.batch
    n = cfg.rotary_dim or cfg.head_dim
    m = cfg.magnitude if cfg.magnitude > 0 else 1.0
    for call, sign in ((rot.forward, 1.0), (rot.backward, -1.0)):
        for x, got in zip((q, k), call(q, k, q_start=_start(starts))):
            want, bound = R.turn(x, at, rot.freqs.tolist(), cfg.interleaved, m, sign)
            R.check("turned", got, want, bound)
            assert torch.equal(got[..., n:], x[..., n:])
    return q, k, rot


SHAPES = [(1, 1, 1, 64), (2, 3, 4, 128), (3, 50, 5, 80), (1, 7, 2, 96), (2, 9, 3, 256), (2, 5, 2, 512),
          (4, 33, 12, 64), (1, 1000, 3, 64), (5, 4, 2, 2), (2, 3, 3, 14), (1, 2100, 2, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shapes(shape, interleaved, dtype):
    _check(C(*shape, dtype=dtype, interleaved=interleaved), 1)
    _check(C(shape[0], shape[1], 6, shape[3], kv_heads=2, dtype=dtype, interleaved=interleaved), 2,
           [3 + 100 * b for b in range(shape[0])])


@pytest.mark.gpu
@pytest.mark.parametrize("head_dim,rotary_dim", [(64, 2), (64, 30), (64, 48), (65, 64), (80, 20), (81, 6),
                                                 (7, 4), (128, 126), (129, 128), (256, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_a_head(head_dim, rotary_dim, interleaved, dtype):
    _check(C(2, 5, 3, head_dim, rotary_dim=rotary_dim, dtype=dtype, interleaved=interleaved,
             magnitude=1.3), 3, [11, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("start", [-5, -2 ** 31, 2 ** 20, 2 ** 24 + 1, 2 ** 31 - 1 - 40])
@pytest.mark.parametrize("scaling", ["none", "linear", "parts"])
def test_far_positions(start, scaling):
    """Angles of up to 2^31 radians are known to 2^-20 of one (the bound)."""
    _check(C(2, 40, 2, 64, dtype="f32", base=5e5, scaling=scaling, factor=8.0, original_len=8192), 4,
           [start, 0])


@pytest.mark.gpu
def test_positions_past_32_bits():
    """The last position of a sequence that starts at the largest start."""
    _check(C(1, 9, 1, 64, dtype="f32"), 5, [2 ** 31 - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_own_frequencies_and_nothing_to_turn(interleaved):
    q, k, rot = _check(C(2, 6, 2, 32, interleaved=interleaved), 6)
    rot.freqs = torch.zeros_like(rot.freqs)
    a, b = rot.forward(q, k)
    assert torch.equal(a, q) and torch.equal(b, k)
    rot.freqs = torch.full_like(rot.freqs, math.pi / 2)     # quarter turns, 6 positions
    f = rot.freqs.tolist()
    for x, got in zip((q, k), rot.forward(q, k)):
        R.check("turned", got, *R.turn(x, [0, 0], f, interleaved, 1.0))
    rot.freqs = rot.freqs[:3]
    with pytest.raises(abft.AbftError):
        rot.forward(q, k)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_there_and_back(dtype, interleaved):
    """The backward is the transpose: <turn(x), g> = <x, back(g)> to the roundings of
    both results."""
    cfg = C(2, 33, 3, 80, rotary_dim=60, dtype=dtype, interleaved=interleaved, magnitude=1.1)
    (x, k, _), (g, gk, _) = _inputs(cfg, 7), _inputs(cfg, 8)
    rot = abft.Rotary(cfg)
    st = _start([5, 70000])
    y, gx = rot.forward(x, k, q_start=st)[0], rot.backward(g, gk, q_start=st)[0]
    one, two = (y.double() * g.double()), (x.double() * gx.double())
    bound = (R.half_step(DT[dtype]) + 2 ** -20) * 1.3 * (one.abs().sum() + two.abs().sum())
    assert (one.sum() - two.sum()).abs() <= bound


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("head_dim,rotary_dim", [(64, 64), (72, 50)])
def test_views_and_in_place(dtype, interleaved, head_dim, rotary_dim):
    """Views of a packed projection at an odd element, heads in front of tokens; in
    place, what lies between stays."""
    cfg = C(2, 9, 4, head_dim, kv_heads=2, rotary_dim=rotary_dim, dtype=dtype, interleaved=interleaved)
    q, k, v = _inputs(cfg, 9)
    rot = abft.Rotary(cfg)
    st = _start([4, 900])
    want = rot.forward(q, k, q_start=st)
    flat = torch.full((1 + 2 * 9 * 9 * head_dim,), 3.0, dtype=DT[dtype], device="cuda")
    packed = flat[1:].view(2, 9, 9, head_dim)
    pq, pk = packed[:, :, :4], packed[:, :, 5:7]
    pq.copy_(q), pk.copy_(k)
    got = rot.forward(pq, pk, q_start=st)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    rot.forward(pq, pk, q_start=st, Q_out=pq, K_out=pk)
    assert torch.equal(pq, want[0]) and torch.equal(pk, want[1])
    pq.fill_(3.0), pk.fill_(3.0)
    assert (flat == 3.0).all()
    qt = torch.empty((2, 4, 9, head_dim), dtype=DT[dtype], device="cuda").transpose(1, 2)
    rot.forward(q, k, q_start=st, Q_out=qt)
    assert torch.equal(qt, want[0])
    rep = q[:, :1].expand(2, 9, 4, head_dim)
    assert torch.equal(rot.forward(rep, k, q_start=st)[0], rot.forward(rep.contiguous(), k, q_start=st)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,starts", [(1, [0, 19, 7]), (3, [0, 17, 18]), (20, [0, 0, 5]),
                                           (5, [-2, -9, 25]), (2, None)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(tokens, starts, dtype, interleaved):
    """New rows go where their positions say, those without a place are left out,
    and no other row is touched."""
    cap, cfg = 20, C(3, tokens, 6, 64, kv_heads=2, rotary_dim=40, dtype=dtype, interleaved=interleaved)
    print(f"[case] append {cfg} {starts}", flush=True)
    q, k, v = _inputs(cfg, 10)
    rot = abft.Rotary(cfg)
    tq, tk = rot.forward(q, k, q_start=_start(starts))
    for order in (1, 2):       # tokens in front of heads in the cache, and behind them
        shape = [3, cap, 2, 64]
        shape[1], shape[order] = shape[order], shape[1]
        caches = [torch.full(shape, float(5 + i), dtype=DT[dtype], device="cuda").transpose(1, order)
                  for i in range(2)]
        want = [c.clone() for c in caches]
        for b in range(3):
            for i in range(tokens):
                at = (starts[b] if starts else 0) + i
                if 0 <= at < cap:
                    want[0][b, at], want[1][b, at] = tk[b, i], v[b, i]
        out = rot.append(q, k, v, *caches, q_start=_start(starts))
        assert torch.equal(out, tq)
        assert all(torch.equal(a, b) for a, b in zip(caches, want))
    q2 = q.clone()
    rot.append(q2, k, v, *caches, q_start=_start(starts), Q_out=q2)
    assert torch.equal(q2, tq)
    empty = torch.empty((3, 0, 2, 64), dtype=DT[dtype], device="cuda")
    assert torch.equal(rot.append(q, k, v, empty, empty, q_start=_start(starts)), tq)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,rotary_dim", [(3, 0, 32), (0, 2, 32), (3, 2, 0), (0, 2, 0)])
def test_c_calls_without_queries_keys_or_turned_dims(heads, kv_heads, rotary_dim):
    cfg = C(2, 5, 3, 40, kv_heads=2)
    q, k, v = _inputs(cfg, 13)
    c = abft.RotaryConfigC(2, 5, heads, kv_heads, 40, rotary_dim, 0, 0, 1.0)
    rot = abft.Rotary(C(2, 5, 3, 40, kv_heads=2, rotary_dim=32))
    tq, tk = rot.forward(q, k)
    if rotary_dim == 0:
        tq, tk = q, k
    at = lambda t: ctypes.byref(abft.CrossTensor(t.data_ptr(), *t.stride()[:3]))
    null = ctypes.byref(abft.CrossTensor(None, 0, 0, 0))
    freqs = rot.freqs.data_ptr() if rotary_dim else None
    qo, ko, vo = (torch.full_like(t, 7.0) for t in (q, k, v))
    stream = torch.cuda.current_stream().cuda_stream
    args = [at(t) if n else null for t, n in ((q, heads), (k, kv_heads))]
    outs = [at(t) if n else null for t, n in ((qo, heads), (ko, kv_heads))]
    assert abft._lib.attn_rotary(c, 0, *args, freqs, None, *outs, stream) == 0
    assert torch.equal(qo, tq if heads else torch.full_like(q, 7.0))
    assert torch.equal(ko, tk if kv_heads else torch.full_like(k, 7.0))
    qo.fill_(7.0), ko.fill_(7.0)
    args.append(at(v) if kv_heads else null)
    outs.append(at(vo) if kv_heads else null)
    assert abft._lib.attn_rotary_append(c, *args, freqs, None, 5, *outs, stream) == 0
    assert torch.equal(qo, tq if heads else torch.full_like(q, 7.0))
    assert torch.equal(ko, tk if kv_heads else torch.full_like(k, 7.0))
    assert torch.equal(vo, v if kv_heads else torch.full_like(v, 7.0))


@pytest.mark.gpu
def test_python_refusals():
    rot = abft.Rotary(C(2, 3, 4, 16, kv_heads=2))
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    q, k, kc, vc = z(2, 3, 4, 16), z(2, 3, 2, 16), z(2, 9, 2, 16), z(2, 9, 2, 16)
    for call in (lambda: rot.forward(q, q), lambda: rot.forward(q.float(), k), lambda: rot.forward(q.cpu(), k),
                 lambda: rot.forward(q[:, :2], k), lambda: rot.forward(q.transpose(2, 3), k),
                 lambda: rot.forward(z(2, 3, 4, 32)[..., ::2], k),
                 lambda: rot.forward(q, k, q_start=_start([1, 2, 3])),
                 lambda: rot.forward(q, k, q_start=_start([1, 2]).long()),
                 lambda: rot.forward(q, k, Q_out=q[:, :1].expand(2, 3, 4, 16)),
                 lambda: rot.forward(q, q[:, :, :2], Q_out=q),                 # keys in what is written
                 lambda: rot.append(q, k, k, kc, kc), lambda: rot.append(q, k, k, kc, vc[:, :8]),
                 lambda: rot.append(q, kc[:, :3], k, kc, vc), lambda: rot.append(q, k, k, kc.float(), vc)):
        with pytest.raises(abft.AbftError):
            call()


@pytest.mark.gpu
def test_a_long_cache():
    """Rows further than 2^32 bytes into a cache."""
    cfg = C(1, 2, 4, 128, kv_heads=2, dtype="f32")
    q, k, v = _inputs(cfg, 11)
    rot = abft.Rotary(cfg)
    cap = 5 * 2 ** 20
    kc = torch.zeros((1, cap, 2, 128), device="cuda")        # 5 GiB
    vc = torch.zeros((1, cap, 2, 128), device="cuda")
    st = _start([cap - 2])
    _, tk = rot.forward(q, k, q_start=st)
    rot.append(q, k, v, kc, vc, q_start=st)
    assert torch.equal(kc[:, -2:], tk) and torch.equal(vc[:, -2:], v)
    assert not kc[:, :-2].any() and not vc[:, :-2].any()


@pytest.mark.gpu
def test_captured_calls_follow_their_positions():
    cfg = C(4, 1, 8, 64, kv_heads=2)
    q, k, v = _inputs(cfg, 12)
    rot = abft.Rotary(cfg)
    kc, vc = (torch.zeros((4, 30, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st, out = _start([0, 3, 5, 20]), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rot.append(q, k, v, kc, vc, q_start=st, Q_out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rot.append(q, k, v, kc, vc, q_start=st, Q_out=out)
    for _ in range(4):
        st += 1
        ek, ev = kc.clone(), vc.clone()
        want = rot.append(q, k, v, ek, ev, q_start=st)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(kc, ek) and torch.equal(vc, ev)
