"""Clipping where the factor, or the norm, leaves the range of fp32."""
import math

import pytest
import torch

from paper_2410_11720_amd import abft


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("std,max_norm", [(2.0 ** 125, 1.0), (2.0 ** 120, 2.0 ** -20),
                                          (2.0 ** 126, 2.0 ** -100), (2.0 ** 100, 2.0 ** -30),
                                          (3.38e38, 1.0), (3.38e38, 1e-60)])
@pytest.mark.parametrize("inplace", [False, True])
def test_factors_below_the_normal_range(dtype, std, max_norm, inplace):
    """Each output is gradient * max_norm / norm, off by three roundings of 64
    bits, three of fp32 and the storage's, and by half a step of the type's
    smallest numbers, though the factor itself is below 2^-126."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    grads = [(torch.rand(n, generator=gen, device="cuda") * 2 - 1) for n in (300000, 77, 5)]
    grads = [(g * std).to(dtype) for g in grads]
    assert all(g.isfinite().all() for g in grads)
    before = [g.double() for g in grads]
    # (squares of 2^250 stay in the range of 64 bits)
    norm = math.sqrt(sum(float((g ** 2).sum()) for g in before))
    out = grads if inplace else [torch.empty_like(g) for g in grads]
    stats = abft.GradientClip(grads).clip(grads, max_norm, out)
    assert stats.nonfinite.item() == 0
    u, least = torch.finfo(dtype).eps / 2, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for b, o in zip(before, out):
        want = b * (max_norm / norm)
        bad = (o.double() - want).abs() > (u + 2.0 ** -22) * want.abs() + least
        assert not bad.any(), (int(bad.sum()), b[bad][0].item(), o[bad][0].item(), want[bad][0].item())
    total = math.sqrt(sum(float((o.double() ** 2).sum()) for o in out))
    # (n elements each off by `least` move the norm by at most least sqrt(n): all of
    # it where max_norm is below the type's smallest number)
    n = sum(o.numel() for o in out)
    assert abs(total - max_norm) <= (u + 2.0 ** -20) * max_norm + least * math.sqrt(n)
    # the norm as fp32 has it: INF past its range, with no element to blame
    as_fp32 = torch.tensor(norm, dtype=torch.float64).float().item()
    assert stats.norm.item() == pytest.approx(as_fp32, rel=2.0 ** -22)
