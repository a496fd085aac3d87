"""Attention over keys of another length in 64 bits, from the definition, with
bounds on what a computation of the stated roundings may be off by.

Roundings of the kernels (u: half a step of the storage type): P and dS enter
the second products in the storage type; O, dQ, dK, dV are stored in it; D is
formed from the stored O. Everything else is fp32 (v = 2^-24): a score's sum of
head_dim products and its few operations up to the exponent, whose absolute error
is the relative error of P; sums over keys or queries in any order."""
import math

import torch

V32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def bucket(rel, buckets, max_distance, bidirectional):
    """In whole numbers: distance n >= e lies in log bucket t or above iff
    (n / e)^f >= (max / e)^t."""
    side = buckets // 2 if bidirectional else buckets
    base = side if bidirectional and rel > 0 else 0
    n = abs(rel) if bidirectional else max(-rel, 0)
    e = side // 2
    if n < e:
        return base + n
    f, t = side - e, 0
    n = min(n, max_distance)
    while t < f - 1 and n ** f >= e ** (f - t - 1) * max_distance ** (t + 1):
        t += 1
    return base + e + t


def reference(Q, K, V, dO=None, bias=None, lens=None, starts=None, causal=False, scale=None,
              max_distance=128, bidirectional=True):
    """Returns {name: (value, bound)} in float64; with dO also the gradients."""
    dtype = Q.dtype
    u = half_step(dtype)
    B, Sq, nh, d = Q.shape
    Sk, kvh = K.shape[1], K.shape[2]
    group = nh // kvh
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    dev = Q.device
    f64 = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)
    out = {k: (f64(B, Sq, nh, d), f64(B, Sq, nh, d)) for k in ("O", "dQ")}
    out.update({k: (f64(B, Sk, kvh, d), f64(B, Sk, kvh, d)) for k in ("dK", "dV")})
    nb = 0 if bias is None else bias.shape[0]
    out["dbias"] = (f64(max(nb, 1), nh), f64(max(nb, 1), nh))
    out["lse"] = (torch.full((B, nh, Sq), -math.inf, dtype=torch.float64, device=dev),
                  f64(B, nh, Sq))
    add = lambda name, at, x: out[name][0].__setitem__(at, out[name][0][at] + x)
    err = lambda name, at, x: out[name][1].__setitem__(at, out[name][1][at] + x)
    table = {}
    for b in range(B):
        n = Sk if lens is None else min(max(int(lens[b]), 0), Sk)
        start = 0 if starts is None else int(starts[b])
        if n == 0 or Sq == 0:
            continue
        rel = torch.arange(n, device=dev)[None, :] - (start + torch.arange(Sq, device=dev))[:, None]
        ok = rel <= 0 if causal else torch.ones_like(rel, dtype=torch.bool)
        if nb:
            lo = int(rel.min())
            key = (lo, int(rel.max()))
            if key not in table:
                table[key] = torch.tensor([bucket(r, nb, max_distance, bidirectional)
                                           for r in range(lo, key[1] + 1)], device=dev)
            which = table[key][rel - lo]
        for h in range(nh):
            q, k, v = Q[b, :, h].double(), K[b, :n, h // group].double(), V[b, :n, h // group].double()
            s = scale * (q @ k.T)
            mag = abs(scale) * (q.abs() @ k.abs().T)
            if nb:
                s = s + bias[:, h].double()[which]
                mag = mag + bias[:, h].double()[which].abs()
            s = s.masked_fill(~ok, -math.inf)
            seen = ok.any(dim=1)
            p = torch.zeros_like(s)
            p[seen] = torch.softmax(s[seen], dim=1)
            out["lse"][0][b, h][seen] = torch.logsumexp(s[seen], dim=1) / math.log(2.0)
            # relative error of P: the exponent's absolute error (head_dim
            # products and 8 more operations on values of at most mag, the
            # maximum or lse among them), and 8 for exp2, sums' scaling, division
            top = (mag * ok).amax(dim=1, keepdim=True)
            es = V32 * ((d + 8) * (mag + top) + 8)
            out["lse"][1][b, h] = V32 * ((d + 8) * 2 * top[:, 0] + n + 8) * 1.5
            pv = p @ v.abs()
            o = p @ v
            add("O", (b, slice(None), h), o)
            err("O", (b, slice(None), h),
                (u + (n + 4) * V32) * pv + 2 * ((p * es) @ v.abs()) + (es * p).sum(1, keepdim=True) * pv
                + u * o.abs())
            if dO is None:
                continue
            g = dO[b, :, h].double()
            dp = g @ v.T
            D = (g * o).sum(1, keepdim=True)
            ds = p * (dp - D)
            e_o = out["O"][1][b, :, h]
            e_D = (g.abs() * (e_o + u * o.abs())).sum(1, keepdim=True)
            e_dp = V32 * (d + 4) * (g.abs() @ v.abs().T + g.abs().matmul(o.abs().T).diagonal()[:, None])
            e_ds = ds.abs() * (u + 2 * es + 4 * V32) + p * (e_D + e_dp) * (1 + 2 * es)
            at, ak = (b, slice(None), h), (b, slice(0, n), h // group)
            dq, dk, dv = scale * (ds @ k), scale * (ds.T @ q), p.T @ g
            add("dQ", at, dq)
            err("dQ", at, scale * ((e_ds + V32 * (n + 4) * ds.abs()) @ k.abs()) + u * dq.abs())
            add("dK", ak, dk)
            err("dK", ak, scale * ((e_ds + V32 * (Sq * group + 4) * ds.abs()).T @ q.abs()))
            add("dV", ak, dv)
            err("dV", ak, (p * (u + 2 * es + V32 * (Sq * group + 4))).T @ g.abs())
            if nb:
                one = lambda x: torch.bincount(which.reshape(-1), weights=x.reshape(-1), minlength=nb)
                add("dbias", (slice(None), h), one(ds))
                err("dbias", (slice(None), h), one(e_ds + V32 * (B * Sq + n) * ds.abs()))
    for k in ("dK", "dV"):
        out[k][1].add_(u * out[k][0].abs())
    return out


def check(got, want, names):
    """Asserts |got - value| <= bound elementwise (and equal infinities)."""
    for name, g in zip(names, got):
        value, bound = want[name]
        g = g.double()
        assert g.shape == value.shape, (name, g.shape, value.shape)
        same = torch.isinf(value) & (g == value)
        off = (g - value).abs()
        bad = ~((off <= bound + 1e-30) | same)
        if bad.any():
            at = bad.nonzero()[0].tolist()
            raise AssertionError(
                f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds, first at {at}: "
                f"{g[tuple(at)].item()} for {value[tuple(at)].item()} +- {bound[tuple(at)].item()}")
