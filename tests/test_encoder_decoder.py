"""The operators as they are used together: an encoder-decoder's attention in
one training step (encoder self attention with a two-sided bias, causal decoder
self attention with a one-sided bias, cross attention to the padded encoder
states), its gradients clipped; and the decoder token by token over a cache."""
import math

import pytest
import torch

import cross_reference as R
from paper_2410_11720_amd import abft

C = abft.CrossConfig
B, NS, NT, NH, D, NB = 2, 90, 70, 4, 64, 16


def _plain(q, k, v, ok, bias=None):
    s = torch.einsum("bihd,bjhd->bhij", q, k) / math.sqrt(D)
    if bias is not None:
        s = s + bias
    s = s.masked_fill(~ok, -math.inf)
    return torch.einsum("bhij,bjhd->bihd", torch.softmax(s, dim=3), v)


def _table(n, two_sided):
    return torch.tensor([[R.bucket(j - i, NB, 32, two_sided) for j in range(n)] for i in range(n)],
                        device="cuda")


@pytest.mark.gpu
def test_training_step_and_clipping():
    """In full precision, against autograd in 64 bits. Each of the nine passes
    sums at most d + n < 2^8 products of values around 1 and exponents below 2^4,
    so it adds less than 2^8 2^4 2^-24 = 2^-12 in relative norm; nine of them 2^-8.8."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    enc, dec = rnd(B, NS, 3, NH, D), rnd(B, NT, 3, NH, D)   # packed projections
    tab_e, tab_d, g = rnd(NB, NH), rnd(NB, NH), rnd(B, NT, NH, D)
    lens = torch.tensor([NS, 53], dtype=torch.int32, device="cuda")

    def att(cfg):
        return abft.CrossAttention(cfg)
    e_att = att(C(B, NS, NS, NH, D, dtype="f32", buckets=NB, max_distance=32))
    d_att = att(C(B, NT, NT, NH, D, dtype="f32", causal=True, buckets=NB, max_distance=32,
                  bidirectional=False))
    x_att = att(C(B, NT, NS, NH, D, dtype="f32"))
    eq, ek, ev = (enc[:, :, i] for i in range(3))
    dq, dk, dv = (dec[:, :, i] for i in range(3))
    e = e_att.forward(eq, ek, ev, bias=tab_e, k_lens=lens)
    d = d_att.forward(dq, dk, dv, bias=tab_d)
    o = x_att.forward(d, e, e, k_lens=lens)
    # backward; gradients of the packed tensors into packed ones
    g_enc, g_dec = torch.empty_like(enc), torch.empty_like(dec)
    gd, gk, gv, _ = x_att.backward(g, d, e, e, o, k_lens=lens)
    ge = gk + gv
    *_, g_te = e_att.backward(ge, eq, ek, ev, e, bias=tab_e, k_lens=lens, dQ=g_enc[:, :, 0],
                              dK=g_enc[:, :, 1], dV=g_enc[:, :, 2])
    *_, g_td = d_att.backward(gd, dq, dk, dv, d, bias=tab_d, dQ=g_dec[:, :, 0],
                              dK=g_dec[:, :, 1], dV=g_dec[:, :, 2])

    leaves = [t.double().requires_grad_() for t in (enc, dec, tab_e, tab_d)]
    xe, xd, te, td = leaves
    seen = (torch.arange(NS, device="cuda") < lens[:, None])[:, None, None, :]
    past = torch.ones((NT, NT), dtype=torch.bool, device="cuda").tril()
    e2 = _plain(xe[:, :, 0], xe[:, :, 1], xe[:, :, 2], seen,
                te[_table(NS, True)].permute(2, 0, 1))
    d2 = _plain(xd[:, :, 0], xd[:, :, 1], xd[:, :, 2], past,
                td[_table(NT, False)].permute(2, 0, 1))
    o2 = _plain(d2, e2, e2, seen)
    o2.backward(g.double())
    got = [g_enc, g_dec, g_te, g_td]
    for a, b in zip([o, *got], [o2.detach(), *(t.grad for t in leaves)]):
        assert (a.double() - b).norm() <= 2 ** -8.8 * b.norm()

    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in got))
    before = [t.clone() for t in got]
    stats = abft.GradientClip(got).clip(got, 1.0)
    assert abs(stats.norm.item() - norm) <= 2 ** -23 * norm and stats.nonfinite.item() == 0
    for a, b in zip(got, before):
        assert ((a - b * stats.coef).abs() <= 2 ** -23 * b.abs() / norm).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decoding_over_a_cache(dtype):
    """A prompt, then token by token: every output lies within the bounds of the
    whole sequence's attention in 64 bits (the same operator, another form)."""
    n0, n, cap = 37, 45, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    q, k, v = rnd(B, n, NH, D), rnd(B, n, 2, D), rnd(B, n, 2, D)
    table = torch.randn((NB, NH), generator=gen, device="cuda")
    kw = dict(kv_heads=2, dtype=dtype, causal=True, buckets=NB, max_distance=32,
              bidirectional=False)
    cache = torch.full((2, B, 2, cap, D), math.nan, dtype=dt, device="cuda")
    kc, vc = cache[0].transpose(1, 2), cache[1].transpose(1, 2)     # [B, cap, 2, D]
    kc[:, :n0], vc[:, :n0] = k[:, :n0], v[:, :n0]
    lens = torch.full((B,), n0, dtype=torch.int32, device="cuda")
    start = torch.zeros((B,), dtype=torch.int32, device="cuda")
    prompt = abft.CrossAttention(C(B, n0, cap, NH, D, **kw), training=False)
    out = [prompt.forward(q[:, :n0], kc, vc, bias=table, k_lens=lens, q_start=start)]
    one = abft.CrossAttention(C(B, 1, cap, NH, D, **kw), training=False)
    start += n0
    for t in range(n0, n):
        kc[:, t], vc[:, t] = k[:, t], v[:, t]
        lens += 1
        out.append(one.forward(q[:, t:t + 1], kc, vc, bias=table, k_lens=lens, q_start=start))
        start += 1
    want = R.reference(q, k, v, bias=table, causal=True, max_distance=32, bidirectional=False)
    R.check([torch.cat(out, dim=1)], want, ["O"])
    with pytest.raises(abft.AbftError):
        one.backward(out[-1], q[:, :1], kc, vc, out[-1], bias=table)
