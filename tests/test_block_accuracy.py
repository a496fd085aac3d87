"""The training step of a decoder block in full precision, result by result, beside a
plain fp32 run of the same: both are held against 64 bits."""
import math

import pytest
import torch

import block_reference as R
from paper_2410_11720_amd import abft
from test_block_together import B, D, H, KVH, NH, RNG, S, _split, _weights

pytestmark = pytest.mark.gpu


def _norm(x, g, b):
    x = x - x.mean(dim=2, keepdim=True)
    return x / (x.square().mean(dim=2, keepdim=True) + 1e-5).sqrt() * g + b


def _turn(t, freqs):
    """Angles in 64 bits whatever t's type, as the operator has them."""
    angle = torch.arange(t.shape[1], device="cuda").double()[:, None] * torch.tensor(
        freqs, dtype=torch.float64, device="cuda")
    cos, sin = (f(angle)[:, None, :].to(t.dtype) for f in (torch.cos, torch.sin))
    a, c = t[..., :D // 2], t[..., D // 2:]
    return torch.cat([a * cos - c * sin, a * sin + c * cos], dim=3)


def _plain(x, w, dy, dh, p, freqs, dtype):
    leaf = {n: t.to(dtype).requires_grad_() for n, t in dict(x=x, **w).items()}
    q, k, v = _split(_norm(leaf["x"], leaf["g1"], leaf["b1"]) @ leaf["wqkv"], S)
    q, k = _turn(q, freqs), _turn(k, freqs)
    k, v = (t.repeat_interleave(NH // KVH, dim=2) for t in (k, v))
    s = (q.transpose(1, 2) @ k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    past = torch.ones((S, S), dtype=torch.bool, device="cuda").tril()
    o = torch.softmax(s.masked_fill(~past, -math.inf), dim=3) @ v.transpose(1, 2).contiguous()
    c = o.transpose(1, 2).flatten(2) @ leaf["wo"]
    if p:
        c = torch.where(R.keep((B, S, H), p, RNG, 5), c * R.scale(p), 0.0)
    h = leaf["x"] + c
    y = _norm(h, leaf["g2"], leaf["b2"])
    (y * dy.to(dtype) + h * dh.to(dtype)).sum().backward()
    return dict(h=h.detach(), y=y.detach(), **{"d" + n: t.grad for n, t in leaf.items()})


@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("seed", [6, 7])
def test_training_step_beside_a_plain_one(p, seed):
    """Each result's error in norm: at most 4 times the plain fp32 run's, whose products
    and sums round as often (attention forms the scores twice and joins partial sums, a
    norm sums its row twice: each less than doubles its count), and one rounding."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = _weights(gen)
    x, dy, dh = (torch.randn((B, S, H), generator=gen, device="cuda") for _ in range(3))
    rng = torch.tensor(RNG, dtype=torch.int64, device="cuda") if p else None
    norm = abft.LayerNorm(abft.NormConfig(B, S, H, dtype="f32"))
    rot = abft.Rotary(abft.RotaryConfig(B, S, NH, D, kv_heads=KVH, dtype="f32"))
    att = abft.CrossAttention(abft.CrossConfig(B, S, S, NH, D, kv_heads=KVH, dtype="f32", causal=True))
    end = abft.ResidualNorm(abft.NormConfig(B, S, H, dtype="f32", dropout=p, site=5))
    a = norm.forward(x, w["g1"], w["b1"])
    q, k, v = _split(a @ w["wqkv"], S)
    q, k = rot.forward(q, k)
    o = att.forward(q, k, v)
    h, y = end.forward(o.flatten(2) @ w["wo"], x, w["g2"], w["b2"], rng=rng)
    dc, dx, dg2, db2 = end.backward(dy, h, w["g2"], dh=dh, rng=rng)
    dwo = o.flatten(2).flatten(0, 1).T @ dc.flatten(0, 1)
    dq, dk, dv, _ = att.backward((dc @ w["wo"].T).unflatten(2, (NH, D)), q, k, v, o)
    dq, dk = rot.backward(dq, dk)
    dqkv = torch.cat([t.flatten(2) for t in (dq, dk, dv)], dim=2)
    dx1, dg1, db1 = norm.backward(dqkv @ w["wqkv"].T, x, w["g1"])
    got = dict(h=h, y=y, dx=dx + dx1, dg1=dg1, db1=db1, dwo=dwo, dg2=dg2, db2=db2,
               dwqkv=a.flatten(0, 1).T @ dqkv.flatten(0, 1))
    freqs = rot.freqs.tolist()
    want, plain = (_plain(x, w, dy, dh, p, freqs, t) for t in (torch.float64, torch.float32))
    assert want.keys() == got.keys()
    for name, value in want.items():
        off = ((got[name].double() - value).norm() / value.norm()).item()
        beside = ((plain[name].double() - value).norm() / value.norm()).item()
        print(f"  {name}: {off:.2e}, plain {beside:.2e}")
        assert off <= 4 * beside + 2.0 ** -24, name
