"""The global gradient norm, and clipping by it, against 64-bit sums."""
import math

import pytest
import torch

from paper_2410_11720_amd import abft

F32, BF16 = torch.float32, torch.bfloat16


def _grads(sizes, seed, dtypes=(F32,), std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=gen, device="cuda") * std).to(dtypes[i % len(dtypes)])
            for i, n in enumerate(sizes)]


def _status(records, n=None, max_norm=1.0, stats=4096, ws=4096, ws_bytes=1 << 20):
    arr = (abft.Grad * max(1, len(records)))(*[abft.Grad(*r, 0) for r in records])
    return abft._lib.clip_gradients(arr, len(records) if n is None else n, max_norm, stats, ws,
                                    ws_bytes, None)


def test_refusals_before_any_launch():
    """Pointers are never followed: the calls return first."""
    ok = (4096, 4096, 10, 1)
    assert _status([ok], n=-1) == -1
    assert _status([(0, 4096, 10, 1)]) == -1 and _status([(4096, 0, 10, 1)]) == -1
    assert _status([(4098, 4098, 10, 1)]) == -1 and _status([(4097, 4098, 10, 0)]) == -1
    assert _status([(4096, 4096, -1, 1)]) == -1 and _status([(4096, 4096, 10, 7)]) == -1
    assert _status([ok], max_norm=-1.0) == -1 and _status([ok], max_norm=math.nan) == -1
    assert _status([ok], stats=None) == -1 and _status([ok], stats=4100) == -1
    assert _status([ok], ws=None) == -1 and _status([ok], ws_bytes=64) == -4
    # the same output twice, and two that share a part, in any order
    assert _status([ok, ok]) == -1
    assert _status([(8192, 8192, 100, 1), (4096, 8188, 2, 1)]) == -1
    # an output on another gradient, on a part of its own, or two exchanged
    assert _status([(4096, 8192, 10, 1), (8192, 16384, 10, 1)]) == -1
    assert _status([(4096, 4100, 10, 1)]) == -1
    assert _status([(4096, 8192, 10, 1), (8192, 4096, 10, 1)]) == -1
    assert _status([(4096, 4096, 10, 1), (4116, 4116, 10, 1)]) == -1
    assert abft._lib.clip_gradients_workspace_bytes(-1) == 0
    assert abft._lib.clip_gradients_workspace_bytes(0) > 0


def _exact(grads, max_norm):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    return norm, (min(1.0, max_norm / norm) if norm else 1.0)


def _check(grads, max_norm, out=None):
    """norm and coef: a few roundings of 64 bits, then one to fp32; an output:
    coef's rounding, the product's and the storage's."""
    before = [g.clone() for g in grads]
    norm, coef = _exact(grads, max_norm)
    clipper = abft.GradientClip(grads)
    clipper.workspace.fill_(255)
    stats = clipper.norm(grads)
    assert abs(stats.norm.item() - norm) <= 2 ** -24 * 1.01 * norm
    assert stats.coef.item() == 1.0 and stats.nonfinite.item() == 0
    clipper.workspace.fill_(255)
    stats = clipper.clip(grads, max_norm, out)
    assert abs(stats.norm.item() - norm) <= 2 ** -24 * 1.01 * norm
    assert abs(stats.coef.item() - coef) <= 2 ** -24 * 1.01 * coef
    assert stats.nonfinite.item() == 0
    for b, g, o in zip(before, grads, grads if out is None else out):
        u = torch.finfo(b.dtype).eps / 2
        want = b.double() * coef
        tiny = torch.finfo(b.dtype).smallest_normal
        assert ((o.double() - want).abs() <= (2 ** -23 * 1.01 + u) * want.abs() + tiny).all()
        if out is not None:
            assert torch.equal(b, g)


SIZES = [[1], [16384], [16385, 16383], [7, 0, 1, 100003, 64, 0], [0], [], [3] * 300,
         [1000 + 37 * i for i in range(113)], [40_000_000, 5]]


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{sum(s)}")
@pytest.mark.parametrize("dtypes", [(F32,), (BF16,), (F32, BF16)], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_norm_and_clip(sizes, dtypes, max_norm):
    grads = _grads(sizes, 4, dtypes)
    _check([g.clone() for g in grads], max_norm)
    _check(grads, max_norm, [torch.empty_like(g) for g in grads])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_any_alignment(dtype):
    """Parts of one buffer at odd elements; what lies between them stays."""
    flat = _grads([70000], 2, (dtype,))[0]
    keep = flat.clone()
    cuts = [(1, 20000), (20003, 20004), (20009, 60001)]
    _check([flat[a:b] for a, b in cuts], 1.0, [torch.empty_like(flat[a:b]) for a, b in cuts])
    _check([flat[a:b] for a, b in cuts], 1.0)
    rest = torch.ones(70000, dtype=torch.bool, device="cuda")
    for a, b in cuts:
        rest[a:b] = False
    assert torch.equal(flat[rest], keep[rest])


@pytest.mark.gpu
@pytest.mark.parametrize("std", [1e30, 1e-30, 1e-36])
def test_extreme_magnitudes(std):
    _check(_grads([5000, 300], 3, (F32,), std), std)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_nonfinite_gradients_are_left_alone(dtype, bad):
    grads = _grads([40000, 9], 6, (dtype,))
    grads[0][39999] = bad
    grads[1][4] = bad
    before = [g.clone() for g in grads]
    clipper = abft.GradientClip(grads)
    out = [torch.zeros_like(g) for g in grads]
    for target in (out, None):
        stats = clipper.clip(grads, 1.0, target)
        assert stats.nonfinite.item() == 2 and stats.coef.item() == 1.0
        norm = stats.norm.item()
        assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
        for g, b, o in zip(grads, before, out):
            assert torch.equal(g.nan_to_num(5.0), b.nan_to_num(5.0))
            assert torch.equal(o.nan_to_num(5.0), b.nan_to_num(5.0))


@pytest.mark.gpu
def test_zero_gradients_and_zero_norm():
    grads = [torch.zeros(100, device="cuda")]
    stats = abft.GradientClip(grads).clip(grads, 1.0)
    assert stats.norm.item() == 0 and stats.coef.item() == 1.0
    grads = [torch.ones(100, device="cuda")]
    stats = abft.GradientClip(grads).clip(grads, 0.0)
    assert stats.coef.item() == 0.0 and (grads[0] == 0).all()


@pytest.mark.gpu
def test_runs_repeat_and_captured_calls_replay():
    sizes = [100000, 33, 70000]
    grads = _grads(sizes, 1)
    out = [torch.empty_like(g) for g in grads]
    clipper = abft.GradientClip(grads)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        clipper.clip(grads, 1.0, out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        clipper.clip(grads, 1.0, out)
    for seed in (11, 12, 13):
        for g, f in zip(grads, _grads(sizes, seed)):
            g.copy_(f)
        clipper.clip(grads, 1.0, out)
        want = [o.clone() for o in out]
        raw = clipper.stats.raw.clone()
        for o in out:
            o.fill_(math.nan)
        clipper.stats.raw.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(raw, clipper.stats.raw)


@pytest.mark.gpu
def test_python_refusals():
    g = torch.ones(8, device="cuda")
    clipper = abft.GradientClip([g])
    for grads, out in (([g, g], None), ([g.half()], None), ([g.cpu()], None),
                       ([torch.ones((8, 8), device="cuda")[:, 0]], None), ([g], [g.bfloat16()]),
                       ([g], [g[:4]]), ([g], [])):
        with pytest.raises(abft.AbftError):
            clipper.clip(grads, 1.0, out)
