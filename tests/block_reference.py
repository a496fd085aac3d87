"""Layer norm, dropout and rotary positions from their definitions: values in 64
bits and how far the kernels' may lie from them.

Bounds count roundings of fp32 (U, half a step) and one of the storage type. A sum
over a row passes at most 24 additions in a lane, 6 between lanes and 16 between
waves: K = 46 roundings of the terms' absolute sum."""
import math

import numpy as np
import torch

U = 2.0 ** -24
K = 46


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- the generator, in plain whole numbers ---------------------------------------

def philox(ctr, key):
    """Philox4x32-10 on arrays of uint64 that hold 32 bits."""
    m = np.uint64(0xFFFFFFFF)
    s = np.uint64(32)
    c = [np.asarray(x, dtype=np.uint64) for x in ctr]
    k = [int(x) for x in key]
    for _ in range(10):
        p0 = c[0] * np.uint64(0xD2511F53)
        p1 = c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> s) ^ c[1] ^ np.uint64(k[0]), p1 & m, (p0 >> s) ^ c[3] ^ np.uint64(k[1]), p0 & m]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def draws(seed, offset, site, rows, cols):
    """[rows, cols] of 16-bit draws."""
    chunk = np.arange((cols + 7) // 8, dtype=np.uint64)[None, :]
    row = np.arange(rows, dtype=np.uint64)[:, None]
    full = np.zeros((rows, chunk.shape[1]), dtype=np.uint64)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    words = philox((full + chunk + np.uint64(site * 2 ** 13), full + row,
                    full + np.uint64(offset % 2 ** 32), full + np.uint64(offset >> 32)),
                   (seed % 2 ** 32, seed >> 32))
    u = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    return u.reshape(rows, -1)[:, :cols].astype(np.int64)


def threshold(p):
    return math.floor(65536 * p + 0.5)


def scale(p):
    t = threshold(p)
    return 0.0 if t == 65536 else 65536 / (65536 - t)


def keep(shape, p, rng, site):
    """[batch, tokens, cols] truth values on the GPU: what stays."""
    B, S, H = shape
    seed, offset = rng
    u = draws(seed, offset, site, B * S, H).reshape(B, S, H)
    return torch.from_numpy(u >= threshold(p)).cuda()


def dropped(x, kept, p):
    """Dropout to the bit: one fp32 product an element (before the storage)."""
    return torch.where(kept, x.float() * np.float32(scale(p)).item(), torch.zeros_like(x.float()))


# ---- layer norm --------------------------------------------------------------------

def valid_rows(shape, lens):
    B, S, _ = shape
    if lens is None:
        return torch.ones((B, S, 1), dtype=torch.bool, device="cuda")
    return (torch.arange(S, device="cuda").view(1, -1, 1) < lens.view(-1, 1, 1))


def norm(h, weight, bias, eps, lens, out_dtype):
    """y and its bound, and for the backward (xh, its bound, r). h as stored."""
    ok = valid_rows(h.shape, lens)
    x = torch.where(ok, h.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    w = torch.ones(h.shape[2], dtype=torch.float64, device="cuda") if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    mean = x.mean(dim=2, keepdim=True)
    r = 1 / ((x - mean).square().mean(dim=2, keepdim=True) + eps).sqrt()
    xh = (x - mean) * r
    # mean: its own rounding, and K of the mean absolute difference (at most 1 / r);
    # 1 / deviation: half of a sum of squares' K + 4 roundings and three more
    e = U * (mean.abs() * r + (K + 2) + (K / 2 + 8) * xh.abs())
    y = xh * w + b
    bound = w.abs() * e + 4 * U * ((xh * w).abs() + b.abs()) + half_step(out_dtype) * y.abs() * 1.01
    zero = torch.zeros_like(y)
    return torch.where(ok, y, zero), torch.where(ok, bound, zero), (xh, e, r, w, ok)


def norm_backward(dy, dh, saved, out_dtype):
    """dict of (value, bound): the gradient of h, dweight, dbias."""
    xh, e, r, w, ok = saved
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    dy = torch.where(ok, dy.double(), zero)
    g = dy * w
    mean = lambda t: t.mean(dim=2, keepdim=True)
    c1, c2 = mean(g), mean(g * xh)
    dx = r * (g - c1 - xh * c2)
    e1 = (K + 3) * U * mean(g.abs())
    e2 = (K + 4) * U * mean((g * xh).abs()) + mean(g.abs() * e)
    size = g.abs() + c1.abs() + (xh * c2).abs()
    bound = r * (e1 + xh.abs() * e2 + c2.abs() * e + (K / 2 + 16) * U * size)
    if dh is not None:
        dh = torch.where(ok, dh.double(), zero)
        dx = dx + dh
        bound = bound + 2 * U * (dh.abs() + dx.abs())
    bound = torch.where(ok, bound, zero)
    rows = dy.shape[0] * dy.shape[1]
    adds = rows / 128 + 100       # rows of a workgroup, its slots, the join
    total = lambda t: t.sum(dim=(0, 1))
    dw = total(dy * xh)
    dw_bound = total(dy.abs() * e) + (adds + 2) * U * total((dy * xh).abs())
    db = total(dy)
    return dict(dh=(torch.where(ok, dx, zero), bound),
                dweight=(dw, dw_bound), dbias=(db, adds * U * total(dy.abs())))


def stored(value, bound, dtype):
    """The bound with the rounding to storage (values and bounds in 64 bits)."""
    return bound + half_step(dtype) * 1.01 * (value.abs() + bound) + torch.finfo(dtype).smallest_normal


def check(name, got, want, bound):
    assert torch.isfinite(want).all() and got.shape == want.shape, name
    err = (got.double() - want).abs()
    tiny = torch.finfo(got.dtype).smallest_normal
    bad = ~(err <= bound + tiny)
    assert not bad.any(), (name, int(bad.sum()), float((err / (bound + tiny)).max()))


# ---- rotary positions --------------------------------------------------------------

def turn(x, starts, freqs, interleaved, magnitude, sign=1.0):
    """x [batch, tokens, heads, dim] turned, in 64 bits, and the bound of its
    result in x's type. The angle is known to one rounding of half a turn and 2^-51 of
    all turns, its functions to 4 units in their last place (8 half steps)."""
    n = 2 * len(freqs)
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    pos = (torch.tensor(starts, dtype=torch.float64, device="cuda").view(-1, 1)
           + torch.arange(x.shape[1], device="cuda"))
    angle = sign * pos[:, :, None, None] * f
    err = 2 * math.pi * 0.5 * U + angle.abs() * 2.0 ** -51 + 8 * U + 4 * U
    cos, sin = torch.cos(angle) * magnitude, torch.sin(angle) * magnitude
    t = x.double()
    out, bound = t.clone(), torch.zeros_like(t)
    first = slice(0, n, 2) if interleaved else slice(0, n // 2)
    second = slice(1, n, 2) if interleaved else slice(n // 2, n)
    a, c = t[..., first], t[..., second]
    size = magnitude * (a.abs() + c.abs())
    for at, v in ((first, a * cos - c * sin), (second, a * sin + c * cos)):
        out[..., at] = v
        bound[..., at] = size * err
    bound[..., :n] = stored(out, bound, x.dtype)[..., :n]
    return out, bound
