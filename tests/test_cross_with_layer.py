"""The protected layer and what stands beside it in one step: an encoder layer
under checksums, cross attention to its output, the gradients back through both,
clipped; and keys and values guarded by checksums while they are stored."""
import math

import pytest
import torch

from paper_2410_11720_amd import abft

pytestmark = pytest.mark.gpu

B, S, T, H, NH = 2, 128, 70, 256, 4
D = H // NH


def test_step_through_layer_and_cross_attention():
    """Gradients of all weights against autograd in 64 bits. In bf16 a result
    passes at most 16 roundings on its way (projections, scores, weights, products,
    outputs, forward and backward), each of relative norm u = 2^-8 at most, either
    way: 4 u in root mean square; 8 u is allowed."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda std, *s: (torch.randn(s, generator=gen, device="cuda") * std).bfloat16()
    x, queries, g = rnd(1.0, B, S, H), rnd(1.0, B, T, NH, D), rnd(1.0, B, T, NH, D)
    wqkv, wo, wkv = rnd(H ** -0.5, H, 3 * H), rnd(H ** -0.5, H, H), rnd(H ** -0.5, H, 2 * H)
    lens = torch.tensor([S, 77], dtype=torch.int32, device="cuda")

    layer = abft.ProtectedAttention(abft.LayerConfig(B, S, H, NH, block_rows=64))
    cross = abft.CrossAttention(abft.CrossConfig(B, T, S, NH, D))
    e = layer.forward(x, wqkv, wo)
    kv = torch.matmul(e.view(-1, H), wkv).view(B, S, 2, NH, D)
    o = cross.forward(queries, kv[:, :, 0], kv[:, :, 1], k_lens=lens)
    dkv = torch.empty_like(kv)
    cross.backward(g, queries, kv[:, :, 0], kv[:, :, 1], o, k_lens=lens, dK=dkv[:, :, 0],
                   dV=dkv[:, :, 1])
    dkv = dkv.view(-1, 2 * H)
    dwkv = torch.matmul(e.view(-1, H).float().t().contiguous(), dkv.float())
    de = torch.matmul(dkv, wkv.t().contiguous()).view(B, S, H)
    _, dwqkv, dwo = layer.backward(de, x, wqkv, wo)
    assert abft.read_report(layer.report)["n_events"] == 0
    assert abft.read_report(layer.report_bwd)["n_events"] == 0

    leaves = [w.double().requires_grad_() for w in (wqkv, wo, wkv)]
    w1, w2, w3 = leaves
    q2, k2, v2 = (t.view(B, S, NH, D) for t in (x.double() @ w1).split(H, dim=2))
    att = torch.softmax(torch.einsum("bihd,bjhd->bhij", q2, k2) / math.sqrt(D), dim=3)
    e2 = torch.einsum("bhij,bjhd->bihd", att, v2).reshape(B, S, H) @ w2
    k3, v3 = (e2 @ w3).view(B, S, 2, NH, D).unbind(2)
    s = torch.einsum("bihd,bjhd->bhij", queries.double(), k3) / math.sqrt(D)
    s = s.masked_fill((torch.arange(S, device="cuda") >= lens[:, None])[:, None, None], -math.inf)
    o2 = torch.einsum("bhij,bjhd->bihd", torch.softmax(s, dim=3), v3)
    o2.backward(g.double())
    grads = [dwqkv, dwo, dwkv]
    for got, want in zip([o, *grads], [o2.detach(), *(w.grad for w in leaves)]):
        assert (got.double() - want).norm() <= 8 * 2.0 ** -8 * want.norm()

    # the end of the step: one norm over the layer's gradients and the projection's
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    before = [t.clone() for t in grads]
    clipper = abft.GradientClip(grads)
    stats = clipper.clip(grads, 0.5 * norm)
    assert stats.nonfinite.item() == 0 and abs(stats.norm.item() - norm) <= 2.0 ** -23 * norm
    for a, b in zip(grads, before):
        assert ((a - 0.5 * b).abs() <= 2.0 ** -22 * b.abs()).all()
    # a fault that no check has seen: counted, and the gradients left alone
    dwo[3, 5] = math.nan
    before = [t.clone() for t in grads]
    stats = clipper.clip(grads, 0.5 * norm)
    assert stats.nonfinite.item() == 1 and stats.coef.item() == 1
    assert all(torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9)) for a, b in zip(grads, before))


@pytest.mark.parametrize("dtype,bits", [("bf16", 3), ("f32", 3)])
@pytest.mark.parametrize("fault", [math.inf, math.nan, 1e12])
def test_stored_keys_and_values_under_checksums(dtype, bits, fault):
    """Projected keys and values of one packed tensor, whose views the attention
    reads, under row and column checksums. Values are multiples of 2^-3 below 2^3:
    every checksum is exact, and so is what is rebuilt from it."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    cfg = abft.CrossConfig(B, T, S, NH, D, dtype=dtype)
    kv = torch.randn((B, S, 2, NH, D), generator=gen, device="cuda").clamp(-7, 7)
    kv = ((kv * 2 ** bits).round() / 2 ** bits).to(cfg.torch_dtype)
    q = torch.randn((B, T, NH, D), generator=gen, device="cuda").to(cfg.torch_dtype)
    lens = torch.tensor([S, 77], dtype=torch.int32, device="cuda")
    att = abft.CrossAttention(cfg, training=False)
    clean = att.forward(q, kv[:, :, 0], kv[:, :, 1], k_lens=lens)

    cols, R = 2 * H, 64
    code = abft.FP32 if dtype == "f32" else abft.BF16
    col = torch.empty((B, S // R, 2, cols), dtype=torch.float32, device="cuda")
    row = torch.empty((B, S, cols // R, 2), dtype=torch.float32, device="cuda")
    abft.encode_checksums(kv, code, B, S, cols, cols, S * cols, R, R, col, row)
    kept = kv.clone()
    kv[0, 40, 0, 2, 7] = fault           # a key
    kv[1, 70, 1, 1, 60] = fault          # a value
    bad = att.forward(q, kv[:, :, 0], kv[:, :, 1], k_lens=lens)
    assert not torch.equal(bad, clean)
    report = abft.new_report(64)
    abft.verify_and_correct(kv, code, B, S, cols, cols, S * cols, R, R, col, row, 1e10, 1e5, 0.0,
                            abft.OP_ID["CL"], report)
    got = abft.read_report(report)
    assert got["n_events"] == 2 and got["n_uncorrectable"] == 0
    assert torch.equal(kv, kept)
    assert torch.equal(att.forward(q, kv[:, :, 0], kv[:, :, 1], k_lens=lens), clean)
