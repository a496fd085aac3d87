"""How near attention over keys of another length comes to its definition: the
norm of each result's error against what its roundings amount to when they fall
either way (root mean squares), where tests/cross_reference.py bounds every
element by their worst sum. A bias gradient, a sum of many dS of either sign, is
held by this only.

Roundings (v: half a step of fp32, u: of the storage type), each independent:
 s       sqrt(d) + 8 of v, of at most m = scale |q| . |k| + |bias|, and as many of
         the row's largest m in the lse
 P       the absolute error of s, and 8 v (exponential, lse, division)
 dP      sqrt(d) + 4 of v, of |dO| . |v|
 D       summed from P dP: what its row's P and dP are off by
 dS      |dS| times P's, P times dP's and D's
 O, dQ, dK, dV   P and dS rounded to the storage type once for the product, and
         the result: u each
Errors of one row go together (lse, D); those of different rows do not."""
import ctypes
import math

import pytest
import torch

import cross_reference as R
from paper_2410_11720_amd import abft

C = abft.CrossConfig
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
V = 2.0 ** -24
NAMES = ("O", "dQ", "dK", "dV", "dbias")


def expected(q, k, v, g, bias=None, lens=None, starts=None, causal=False, max_distance=128,
             bidirectional=True):
    """{name: (value, root mean square of the error)} in 64 bits."""
    u = torch.finfo(q.dtype).eps / 2
    p_u = u if q.dtype == torch.bfloat16 else 0.0     # (fp32 keeps P and dS)
    B, Sq, nh, d = q.shape
    Sk, kvh = k.shape[1:3]
    scale = d ** -0.5
    f64 = dict(dtype=torch.float64, device=q.device)
    like = {"O": q.shape, "dQ": q.shape, "dK": k.shape, "dV": k.shape}
    if bias is not None:
        like["dbias"] = bias.shape
    val = {n: torch.zeros(s, **f64) for n, s in like.items()}
    var = {n: torch.zeros(s, **f64) for n, s in like.items()}
    for b in range(B):
        n = Sk if lens is None else min(max(lens[b], 0), Sk)
        start = 0 if starts is None else starts[b]
        rel = torch.arange(n, device=q.device)[None] - (start + torch.arange(Sq, device=q.device))[:, None]
        ok = rel <= 0 if causal else torch.ones_like(rel, dtype=torch.bool)
        if n == 0:
            continue
        if bias is not None:
            lo, hi = int(rel.min()), int(rel.max())
            which = torch.tensor([R.bucket(t, bias.shape[0], max_distance, bidirectional)
                                  for t in range(lo, hi + 1)], device=q.device)[rel - lo]
        for h in range(nh):
            x, y = (slice(None), h), (slice(0, n), h // (nh // kvh))
            qq, gg, kk, vv = q[b][x].double(), g[b][x].double(), k[b][y].double(), v[b][y].double()
            s, m = scale * qq @ kk.T, scale * qq.abs() @ kk.abs().T
            if bias is not None:
                s, m = s + bias[:, h].double()[which], m + bias[:, h].double()[which].abs()
            s = s.masked_fill(~ok, -math.inf)
            seen = ok.any(dim=1)
            p = torch.zeros_like(s)
            p[seen] = torch.softmax(s[seen], dim=1)
            top = (m * ok).amax(dim=1, keepdim=True)
            e_p = V * ((math.sqrt(d) + 8) * (m + top) + 8)          # relative
            o, dp = p @ vv, gg @ vv.T
            e_dp = V * (math.sqrt(d) + 4) * (gg.abs() @ vv.abs().T)
            ds = p * (dp - (gg * o).sum(1, keepdim=True))
            e_d = ((p * e_dp + ds.abs() * e_p) ** 2).sum(1, keepdim=True).sqrt()
            e_ds = ds.abs() * e_p + p * (e_dp + e_d)
            one = V * math.sqrt(n + Sq * nh // kvh)                  # of a sum's own additions
            put = lambda name, at, value, sq: (val[name][b][at].add_(value), var[name][b][at].add_(sq))
            rnd = lambda e, w: (p_u * w) ** 2 + e ** 2
            put("O", x, o, rnd(p * e_p, p) @ vv ** 2 + (one * (p @ vv.abs())) ** 2 + (u * o) ** 2)
            dq = scale * ds @ kk
            put("dQ", x, dq, scale ** 2 * (rnd(e_ds, ds) @ kk ** 2
                                           + (one * (ds.abs() @ kk.abs())) ** 2) + (u * dq) ** 2)
            put("dK", y, scale * ds.T @ qq,
                scale ** 2 * (rnd(e_ds, ds).T @ qq ** 2 + (one * (ds.abs().T @ qq.abs())) ** 2))
            put("dV", y, p.T @ gg, rnd(p * e_p, p).T @ gg ** 2 + (one * (p.T @ gg.abs())) ** 2)
            if bias is not None:
                hot = torch.nn.functional.one_hot(which, bias.shape[0]).double()
                val["dbias"][:, h] += torch.einsum("ij,ijt->t", ds, hot)
                rows = torch.einsum("ij,ijt->it", e_ds, hot)
                var["dbias"][:, h] += (rows ** 2).sum(0) + V ** 2 * (n + Sq) * torch.einsum(
                    "ij,ijt->t", ds ** 2, hot)
    for name in ("dK", "dV"):
        var[name] += (u * val[name]) ** 2
    return {name: (val[name], var[name].sqrt()) for name in val}


def check(got, want, names=NAMES):
    """Norms of the errors, over the tensor and over each head: 2 times the
    expected (entries are many; the roundings are at most what is counted)."""
    for name, x in zip(names, got):
        if x is None:
            continue
        value, rms = want[name]
        err = x.double() - value
        dim = 0 if name == "dbias" else (0, 1, 3)
        off, most = err.norm(), 2 * rms.norm()
        print(f"  {name}: {(off / value.norm()).item():.2e} of at most "
              f"{(most / value.norm()).item():.2e}")
        assert off <= most, (name, off.item(), most.item(), value.norm().item())
        off, most = (err ** 2).sum(dim).sqrt(), 3 * (rms ** 2).sum(dim).sqrt()
        assert (off <= most).all(), (name, off, most)


def _inputs(cfg, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(DT[cfg.dtype])
    kvh = cfg.kv_heads or cfg.heads
    q, g = (rnd(cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim) for _ in range(2))
    k, v = (rnd(cfg.batch, cfg.k_len, kvh, cfg.head_dim) for _ in range(2))
    bias = None
    if cfg.buckets:
        bias = torch.randn((cfg.buckets, cfg.heads), generator=gen, device="cuda")
    return q, k, v, g, bias


def _want(cfg, q, k, v, g, bias, lens, starts):
    return expected(q, k, v, g, bias, lens, starts, cfg.causal, cfg.max_distance,
                    cfg.bidirectional)


ONE = dict(causal=True, bidirectional=False)
CASES = [
    (C(2, 150, 333, 3, 64, buckets=32), [333, 200], None),
    (C(2, 300, 300, 2, 64, buckets=32, **ONE), None, None),
    (C(1, 200, 260, 2, 128, buckets=32), None, None),
    (C(2, 90, 110, 8, 128, kv_heads=2, buckets=64, causal=True), [110, 64], [20, 0]),
    (C(1, 40, 60, 4, 64, buckets=32), None, None),                # one tile of keys
    (C(16, 140, 200, 16, 64, buckets=32), None, None),            # three workgroups a CU
    (C(1, 700, 700, 2, 64, buckets=32, **ONE), None, None),       # axes over workgroups
    (C(1, 600, 40, 8, 64, kv_heads=1, buckets=32), [37], None),
    (C(1, 512, 512, 8, 128, buckets=32), None, None),             # eight waves, 64 keys
    (C(2, 260, 300, 2, 128, kv_heads=1), [300, 40], None),
    (C(2, 200, 333, 12, 64, dtype="f32", buckets=32), [333, 250], None),
    (C(1, 130, 500, 4, 128, dtype="f32", buckets=32), None, None),
    (C(2, 250, 340, 2, 64, dtype="f32", causal=True), [340, 100], [90, -30]),
    (C(3, 70, 60, 2, 128, dtype="f32", buckets=8, **ONE), None, None),
]


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(len(CASES)))
def test_errors_of_all_results(n):
    cfg, lens, starts = CASES[n]
    print(f"[case] {cfg}", flush=True)
    q, k, v, g, bias = _inputs(cfg, 700 + n)
    vec = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    keys = dict(bias=bias, k_lens=vec(lens), q_start=vec(starts))
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v, **keys)
    got = (o, *att.backward(g, q, k, v, o, **keys))
    check(got, _want(cfg, q, k, v, g, bias, lens, starts))


def _record(t):
    return ctypes.byref(abft.CrossTensor(t.data_ptr(), *t.stride()[:3]))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 3, 4, 6, 9])
def test_backward_without_rest(n):
    """The C call with rest = NULL: dQ with D from the rounded O, within the bounds
    of tests/cross_reference.py, which count that; the key pass's D is corrected by
    the row's sum of dS and the rest as accurate as with it. Where a row's keys are
    one tile its D is corrected before dQ too."""
    cfg, lens, starts = CASES[n]
    q, k, v, g, bias = _inputs(cfg, 800 + n)
    vec = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    keys = dict(bias=bias, k_lens=vec(lens), q_start=vec(starts))
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v, **keys)
    at = lambda t: None if t is None else t.data_ptr()
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    db = None if bias is None else torch.empty_like(bias)
    status = abft._lib.attn_cross_backward(
        cfg.to_c(), _record(g), _record(q), _record(k), _record(v), _record(o), at(att.lse), None,
        at(bias), at(keys["k_lens"]), at(keys["q_start"]), _record(dq), _record(dk), _record(dv),
        at(db), at(att.workspace), att.workspace.numel(), torch.cuda.current_stream().cuda_stream)
    assert status == 0
    names = NAMES[2:] if bias is not None else NAMES[2:4]
    check((dk, dv, db), _want(cfg, q, k, v, g, bias, lens, starts), NAMES[2:])
    loose = R.reference(q, k, v, g, bias, keys["k_lens"], keys["q_start"], cfg.causal, None,
                        cfg.max_distance, cfg.bidirectional)
    R.check((dq, dk, dv, db)[:1 + len(names)], loose, ("dQ", *names))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [1, 150])
def test_strides_past_32_bits(dtype, q_len):
    """Sequences, and heads, more than 2^32 bytes apart: inputs and outputs,
    forward (short and tiled) and backward."""
    d, n = 64, 90
    es = DT[dtype].itemsize
    far = (1 << 32) // es + 4096 * 4                # elements
    cfg = C(2, q_len, n, 2, d, dtype=dtype, buckets=32)
    q, k, v, g, bias = _inputs(cfg, 900 + q_len)
    want = _want(cfg, q, k, v, g, bias, None, None)
    for which in ("batch", "head"):
        # eight tensors side by side, the batch (the heads) `far` apart
        room = 2 * max(q_len, n) * d
        buf = torch.empty(far + 8 * room, dtype=DT[dtype], device="cuda")
        views = []
        for i, m in enumerate((q_len, n, n, q_len, q_len, q_len, n, n)):
            st = (far, 2 * d, d, 1) if which == "batch" else (m * d, d, far, 1)
            views.append(buf.as_strided((2, m, 2, d), st, i * room))
        for t, x in zip(views, (q, k, v, g)):
            t.copy_(x)
        fq, fk, fv, fg, fo, dq, dk, dv = views
        att = abft.CrossAttention(cfg)
        att.forward(fq, fk, fv, bias=bias, O=fo)
        *_, db = att.backward(fg, fq, fk, fv, fo, bias=bias, dQ=dq, dK=dk, dV=dv)
        check((fo, dq, dk, dv, db), want)
        for t, x in zip(views, (q, k, v, g)):
            assert torch.equal(t, x)
        del buf, views, fq, fk, fv, fg, fo, dq, dk, dv, t


# ---- host: the backward's refusals ----------------------------------------------------

def _status(cfg, lse=0x60000, bias=0, dbias=0, ws=1 << 40, ws_bytes=1 << 30, rest=0x70000,
            at=0x40000, stride=None, dk=0x2000000, null=None):
    qs = (cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
    ks = (cfg.batch, cfg.k_len, cfg.kv_heads or cfg.heads, cfg.head_dim)

    def t(p, shape, st=None):
        st = st or (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])
        return ctypes.byref(abft.CrossTensor(p, *st))
    args = [t(at, qs), t(0x10000, qs), t(0x20000, ks), t(0x30000, ks), t(0x50000, qs), lse or None,
            rest or None, bias or None, None, None, t(0x1000000, qs), t(dk, ks, stride),
            t(0x3000000, ks), dbias or None]
    if null is not None:
        args[null] = None
    return abft._lib.attn_cross_backward(cfg.to_c(), *args, ws or None, ws_bytes, None)


def test_backward_refuses_before_any_launch():
    """Addresses that are never followed."""
    cfg = C(2, 3, 5, 4, 64)
    biased = C(2, 3, 5, 4, 64, buckets=32)
    assert _status(cfg, lse=0) == -1
    for i in (0, 1, 2, 3, 4, 10, 11, 12):
        assert _status(cfg, null=i) == -1, i
    assert _status(cfg, dbias=0x4000000) == -1 and _status(cfg, bias=0x80000) == -1
    assert _status(biased, bias=0x80000) == -1 and _status(biased, dbias=0x4000000) == -1
    assert _status(cfg, ws=0) == -1 and _status(cfg, ws=(1 << 40) + 8) == -1
    assert _status(cfg, ws_bytes=64) == -4
    assert _status(cfg, rest=0x70008) == -1 and _status(cfg, at=0x40008) == -1
    assert _status(cfg, dk=0) == -1 and _status(cfg, dk=0x2000004) == -1
    assert _status(cfg, stride=(1280, 0, 64)) == -1          # written more than once
    assert _status(cfg, stride=(1280, 256, 60)) == -1
    assert _status(cfg, stride=(2 ** 27, 2 ** 24, 64)) == -2
    assert _status(C(2, 3, 5, 4, 96)) == -2 and _status(C(2, 3, 5, 4, 64, kv_heads=3)) == -1
