"""Layer norm, rotary positions, attention, dropout and the residual as they are
used together: a decoder block's training step, the same block token by token over a
cache, and the protected layer between two norms."""
import math

import numpy as np
import pytest
import torch

import block_reference as R
from paper_2410_11720_amd import abft

B, S, H, NH, KVH, D = 2, 41, 256, 4, 2, 64
RNG = (41, 42)


def _weights(gen, dtype=torch.float32):
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    return dict(g1=1 + 0.2 * rnd(H), b1=0.2 * rnd(H), wqkv=(rnd(H, (NH + 2 * KVH) * D) / 16).to(dtype),
                wo=(rnd(H, H) / 16).to(dtype), g2=1 + 0.2 * rnd(H), b2=0.2 * rnd(H))


def _split(qkv, n):
    q, k, v = qkv.split([NH * D, KVH * D, KVH * D], dim=2)
    return q.unflatten(2, (NH, D)), k.unflatten(2, (KVH, D)), v.unflatten(2, (KVH, D))


def _plain_turn(t, freqs):
    angle = torch.arange(t.shape[1], device="cuda").double()[:, None] * torch.tensor(
        freqs, dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    a, c = t[..., :D // 2], t[..., D // 2:]
    return torch.cat([a * cos - c * sin, a * sin + c * cos], dim=3)


def _plain_norm(x, g, b):
    x = x - x.mean(dim=2, keepdim=True)
    return x / (x.square().mean(dim=2, keepdim=True) + 1e-5).sqrt() * g + b


@pytest.mark.gpu
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_training_step_of_a_block(p):
    """In full precision, against autograd in 64 bits. Each of the twelve passes sums at
    most 2^8 products of values around 1 and exponents below 2^4, so it adds less than
    2^8 2^4 2^-24 = 2^-12 in relative norm; twelve of them 2^-8.4."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    w = _weights(gen)
    x, dy, dh = (torch.randn((B, S, H), generator=gen, device="cuda") for _ in range(3))
    rng = torch.tensor(RNG, dtype=torch.int64, device="cuda") if p else None
    norm = abft.LayerNorm(abft.NormConfig(B, S, H, dtype="f32"))
    rot = abft.Rotary(abft.RotaryConfig(B, S, NH, D, kv_heads=KVH, dtype="f32"))
    att = abft.CrossAttention(abft.CrossConfig(B, S, S, NH, D, kv_heads=KVH, dtype="f32", causal=True))
    end = abft.ResidualNorm(abft.NormConfig(B, S, H, dtype="f32", dropout=p, site=5))

    a = norm.forward(x, w["g1"], w["b1"])
    qkv = a @ w["wqkv"]
    q, k, v = _split(qkv, S)
    rot.forward(q, k, Q_out=q, K_out=k)          # in place, in the packed projection
    o = att.forward(q, k, v)
    c = o.flatten(2) @ w["wo"]
    h, y = end.forward(c, x, w["g2"], w["b2"], rng=rng)
    # backward, into packed gradients
    dc, dx, dg2, db2 = end.backward(dy, h, w["g2"], dh=dh, rng=rng)
    dwo = o.flatten(2).flatten(0, 1).T @ dc.flatten(0, 1)
    dqkv = torch.empty_like(qkv)
    dq, dk, dv = _split(dqkv, S)
    att.backward((dc @ w["wo"].T).unflatten(2, (NH, D)), q, k, v, o, dQ=dq, dK=dk, dV=dv)
    rot.backward(dq, dk, dQ_out=dq, dK_out=dk)
    dwqkv = a.flatten(0, 1).T @ dqkv.flatten(0, 1)
    dx1, dg1, db1 = norm.backward(dqkv @ w["wqkv"].T, x, w["g1"])
    got = [h, y, dx + dx1, dwqkv, dwo, dg1, db1, dg2, db2]

    leaf = {n: t.double().requires_grad_() for n, t in dict(x=x, **w).items()}
    a2 = _plain_norm(leaf["x"], leaf["g1"], leaf["b1"])
    q2, k2, v2 = _split(a2 @ leaf["wqkv"], S)
    freqs = rot.freqs.tolist()
    q2, k2 = _plain_turn(q2, freqs), _plain_turn(k2, freqs)
    k2, v2 = (t.repeat_interleave(NH // KVH, dim=2) for t in (k2, v2))
    s = (q2.transpose(1, 2) @ k2.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    past = torch.ones((S, S), dtype=torch.bool, device="cuda").tril()
    o2 = torch.softmax(s.masked_fill(~past, -math.inf), dim=3) @ v2.transpose(1, 2).contiguous()
    c2 = o2.transpose(1, 2).flatten(2) @ leaf["wo"]
    if p:
        c2 = torch.where(R.keep((B, S, H), p, RNG, 5), c2 * R.scale(p), 0.0)
    h2 = leaf["x"] + c2
    y2 = _plain_norm(h2, leaf["g2"], leaf["b2"])
    (y2 * dy.double() + h2 * dh.double()).sum().backward()
    want = [h2.detach(), y2.detach()] + [leaf[n].grad for n in ("x", "wqkv", "wo", "g1", "b1", "g2", "b2")]
    for g, r in zip(got, want):
        assert (g.double() - r).norm() <= 2 ** -8.4 * r.norm()

    # clipped like the gradients of every other part
    grads = got[2:]
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    stats = abft.GradientClip(grads).clip(grads, 1.0)
    assert abs(stats.norm.item() - norm) <= 2 ** -23 * norm


@pytest.mark.gpu
def test_decoding_over_a_cache():
    """A padded batch of prompts, then token by token: each token's rows are what the
    whole sequence's are, within fp32's roundings (2^-12 a pass, as above; five
    passes)."""
    cap, lens, more = 48, [29, 17], 9
    gen = torch.Generator(device="cuda").manual_seed(4)
    w = _weights(gen)
    x = torch.randn((B, S, H), generator=gen, device="cuda")
    cfg = dict(dtype="f32", causal=True, kv_heads=KVH)

    def block(xs, start, n, cache, counts):
        norm = abft.LayerNorm(abft.NormConfig(B, n, H, dtype="f32"), training=False)
        rot = abft.Rotary(abft.RotaryConfig(B, n, NH, D, kv_heads=KVH, dtype="f32"))
        att = abft.CrossAttention(abft.CrossConfig(B, n, cap, NH, D, **cfg), training=False)
        end = abft.ResidualNorm(abft.NormConfig(B, n, H, dtype="f32"), training=False)
        q, k, v = _split(norm.forward(xs, w["g1"], w["b1"]) @ w["wqkv"], n)
        q = rot.append(q, k, v, *cache, q_start=start)
        o = att.forward(q, *cache, k_lens=counts, q_start=start)
        return end.forward(o.flatten(2) @ w["wo"], xs, w["g2"], w["b2"])[1]
    vec = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")
    whole = [torch.zeros((B, cap, KVH, D), device="cuda") for _ in range(2)]
    want = block(x, vec([0] * B), S, whole, vec([S] * B))

    cache = [torch.full((B, cap, KVH, D), math.nan, device="cuda") for _ in range(2)]
    n = max(lens)
    first = block(x[:, :n].contiguous(), vec([0] * B), n, cache, vec(lens))
    close = lambda a, b: (a.double() - b.double()).norm() <= 5 * 2 ** -12 * b.double().norm()
    for b in range(B):
        assert close(first[b, :lens[b]], want[b, :lens[b]])
    for t in range(more):
        at = [m + t for m in lens]
        xs = torch.stack([x[b, at[b]:at[b] + 1] for b in range(B)])
        y = block(xs, vec(at), 1, cache, vec([m + 1 for m in at]))
        for b in range(B):
            assert close(y[b, 0], want[b, at[b]])
    for b in range(B):
        for got, ref in zip(cache, whole):
            assert close(got[b, :lens[b] + more], ref[b, :lens[b] + more])


@pytest.mark.gpu
def test_protected_layer_between_norms():
    """A norm in front of the protected layer, dropout, residual and norm behind it;
    an INF in its output is corrected before the norm would spread it over a row."""
    import workloads as W
    seq, hid, heads = 128, 256, 4
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    x, dy = rnd(1, seq, hid), rnd(1, seq, hid)
    wqkv, wo = rnd(hid, 3 * hid) * 0.05, rnd(hid, hid) * 0.05
    g, b = torch.ones(hid, device="cuda"), torch.zeros(hid, device="cuda")
    rng = torch.tensor(RNG, dtype=torch.int64, device="cuda")
    norm = abft.LayerNorm(abft.NormConfig(1, seq, hid))
    end = abft.ResidualNorm(abft.NormConfig(1, seq, hid, dropout=0.1))
    layer = abft.ProtectedAttention(abft.LayerConfig(1, seq, hid, heads, causal=True))
    kept = R.keep((1, seq, hid), 0.1, RNG, 0)
    runs = []
    for faults in ([], [W.Fault("O", 0, 0, 77, 100, np.inf)]):
        a = norm.forward(x, g, b)
        o = layer.forward(a, wqkv, wo, abft.faults_to_device(faults) if faults else None)
        h, y = end.forward(o, x, g, b, rng=rng)
        assert torch.equal(h, (x.float() + R.dropped(o, kept, 0.1)).bfloat16())
        do, dx, _, _ = end.backward(dy, h, g, rng=rng)
        da, dwqkv, dwo = layer.backward(do, a, wqkv, wo)
        dx1, dg, db = norm.backward(da, x, g)
        assert len(abft.read_report(layer.report)["events"]) == len(faults)
        runs.append([t.double() for t in (o, h, y, do, dx, da, dwqkv, dwo, dx1, dg, db)])
    for clean, fixed in zip(*runs):
        assert torch.isfinite(clean).all()
        assert (clean - fixed).norm() <= 2 ** -8 * clean.norm()     # (one element, one rounding off)
