"""The encoder-decoder attention step of full precision, result by result, beside
a plain fp32 run of the same step: both are held against 64 bits."""
import math

import pytest
import torch

import cross_reference as R
from paper_2410_11720_amd import abft

pytestmark = pytest.mark.gpu

C = abft.CrossConfig
B, NS, NT, NH, D, NB = 2, 90, 70, 4, 64, 16


def _attend(q, k, v, ok, bias=None):
    s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    if bias is not None:
        s = s + bias
    p = torch.softmax(s.masked_fill(~ok, -math.inf), dim=3)
    return torch.matmul(p, v.transpose(1, 2).contiguous()).transpose(1, 2)


def _table(n, two_sided):
    return torch.tensor([[R.bucket(j - i, NB, 32, two_sided) for j in range(n)] for i in range(n)],
                        device="cuda")


def _plain(enc, dec, tab_e, tab_d, g, lens, dtype):
    leaves = [t.to(dtype).requires_grad_() for t in (enc, dec, tab_e, tab_d)]
    xe, xd, te, td = leaves
    seen = (torch.arange(NS, device="cuda") < lens[:, None])[:, None, None, :]
    past = torch.ones((NT, NT), dtype=torch.bool, device="cuda").tril()
    e = _attend(*xe.unbind(2), seen, te[_table(NS, True)].permute(2, 0, 1))
    d = _attend(*xd.unbind(2), past, td[_table(NT, False)].permute(2, 0, 1))
    o = _attend(d, e, e, seen)
    o.backward(g.to(dtype))
    ge, gd = leaves[0].grad, leaves[1].grad
    return dict(e=e, d=d, o=o, te=te.grad, td=td.grad,
                **{f"enc {n}": ge[:, :, i] for i, n in enumerate("QKV")},
                **{f"dec {n}": gd[:, :, i] for i, n in enumerate("QKV")})


@pytest.mark.parametrize("seed", [3, 4])
def test_training_step_beside_a_plain_one(seed):
    """Each result's error in norm: at most 4 times the plain fp32 run's, whose
    products and sums round as often (a kernel forms the scores twice, joins
    partial sums and takes base-2 exponentials, each less than doubles its count),
    and one rounding of the result."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    enc, dec = rnd(B, NS, 3, NH, D), rnd(B, NT, 3, NH, D)
    tab_e, tab_d, g = rnd(NB, NH), rnd(NB, NH), rnd(B, NT, NH, D)
    lens = torch.tensor([NS, 53], dtype=torch.int32, device="cuda")
    kw = dict(dtype="f32", buckets=NB, max_distance=32)
    e_att = abft.CrossAttention(C(B, NS, NS, NH, D, **kw))
    d_att = abft.CrossAttention(C(B, NT, NT, NH, D, causal=True, bidirectional=False, **kw))
    x_att = abft.CrossAttention(C(B, NT, NS, NH, D, dtype="f32"))
    eq, ek, ev = enc.unbind(2)
    dq, dk, dv = dec.unbind(2)
    e = e_att.forward(eq, ek, ev, bias=tab_e, k_lens=lens)
    d = d_att.forward(dq, dk, dv, bias=tab_d)
    o = x_att.forward(d, e, e, k_lens=lens)
    gd, gk, gv, _ = x_att.backward(g, d, e, e, o, k_lens=lens)
    *ge, te = e_att.backward(gk + gv, eq, ek, ev, e, bias=tab_e, k_lens=lens)
    *gdec, td = d_att.backward(gd, dq, dk, dv, d, bias=tab_d)
    got = dict(e=e, d=d, o=o, te=te, td=td, **{f"enc {n}": t for n, t in zip("QKV", ge)},
               **{f"dec {n}": t for n, t in zip("QKV", gdec)})
    want = _plain(enc, dec, tab_e, tab_d, g, lens, torch.float64)
    plain = _plain(enc, dec, tab_e, tab_d, g, lens, torch.float32)
    for name, value in want.items():
        off = (got[name].double() - value).norm() / value.norm()
        beside = (plain[name].double() - value).norm() / value.norm()
        print(f"  {name}: {off.item():.2e}, plain {beside.item():.2e}")
        assert off <= 4 * beside + 2.0 ** -24, name
