"""What stands between a transformer's attention products, as cases to
measure: layer norm, dropout from a counter-based generator, both with the
residual in one pass, and rotary positions with the append to a cache.

A case's `op`:
  "norm"      LayerNorm.forward
  "norm_step" LayerNorm.forward, then .backward
  "drop"      Dropout.forward, then .backward
  "res"       ResidualNorm.forward (serving: no dropout)
  "res_step"  ResidualNorm.forward, then .backward
  "rot_step"  Rotary.forward, then .backward
  "append"    Rotary.append of new tokens to a cache

`run` in plain torch (`own` false) or through the package's entry points
(`own` true). With n columns a row, w and b the gain and offset:

  norm      y = (x - mean) / sqrt(var + eps) w + b, mean and var of the row;
            rows behind a sequence's length are 0 and give no gradient
  dropout   y = residual + [u >= t] x 65536 / (65536 - t), t = floor(65536 p + 1/2),
            u 16 bits of a Philox4x32-10 word (Salmon, Moraes, Dror, Shaw 2011):
            element (row, col) takes half col % 8 of the eight of counter
            (col / 8 + 2^13 site, row, offset) under the key seed
  residual  h = residual + dropout(x) as it is stored, y = norm(h)
  rotary    token i of sequence b lies at position start_b + i; pair k of a head is
            turned by position f_k and scaled by the magnitude
"""
import math

import torch

own = False


# ---- cases ------------------------------------------------------------------

def _rows(op, batch, tokens, cols, *, dtype="bf16", weight_dtype="f32", lens="full", p=0.0,
          site=0, packed=False, residual=True, name=None):
    c = dict(op=op, batch=batch, tokens=tokens, cols=cols, dtype=dtype, weight_dtype=weight_dtype,
             lens=lens, p=p, site=site, packed=packed, residual=residual)
    if name:
        c["name"] = name
    return c


def _rot(op, batch, tokens, heads, head_dim, *, kv_heads=0, rotary_dim=0, interleaved=False,
         dtype="bf16", base=10000.0, scaling="none", factor=1.0, original_len=2048, magnitude=1.0,
         start=0, capacity=0, name=None):
    c = dict(op=op, batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads or heads,
             head_dim=head_dim, rotary_dim=rotary_dim or head_dim, interleaved=interleaved,
             dtype=dtype, base=base, scaling=scaling, factor=factor, original_len=original_len,
             magnitude=magnitude, start=start, capacity=capacity)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the norm in front of a layer for one decoded token: the smallest call, latency alone
        _rows("norm", 1, 1, 768, name="norm_token"),
        # one norm of the GPT-2 layer's training step
        _rows("norm_step", 8, 1024, 768, name="norm_step"),
        # queries of the same layer normalised by head, views of the packed projection
        _rows("norm_step", 8192, 12, 64, weight_dtype="bf16", packed=True, name="norm_heads_step"),
        # full precision, an odd width, padded sequences
        _rows("norm_step", 3, 333, 1001, dtype="f32", lens="ragged", name="norm_odd_f32"),
        # dropout of an attention output and its residual in a training step
        _rows("drop", 8, 1024, 768, p=0.1, site=1, name="drop_step"),
        # dropout inside the feed-forward part of the decoder of hidden size 4096: the largest
        _rows("drop", 4, 2048, 16384, p=0.1, site=2, residual=False, name="drop_wide"),
        # a batch of decoded tokens: residual and norm, no dropout
        _rows("res", 32, 1, 4096, weight_dtype="bf16", name="res_tokens"),
        # the end of a sublayer of the GPT-2 layer's training step, padded sequences
        _rows("res_step", 8, 1024, 768, p=0.1, site=3, lens="ragged", name="res_step"),
        # the same of one long sequence of a wide decoder
        _rows("res_step", 1, 4096, 5120, weight_dtype="bf16", p=0.1, site=4, name="res_wide_step"),
        # decoded tokens, eight key heads: rotation and append to the cache
        _rot("append", 32, 1, 32, 128, kv_heads=8, capacity=512, start=500, name="append_tokens"),
        # queries and keys of the GPT-2 layer's training step
        _rot("rot_step", 8, 1024, 12, 64, name="rotary_step"),
        # a wide decoder far out in a long context: scaled frequencies, interleaved pairs
        _rot("rot_step", 4, 2048, 40, 128, kv_heads=8, rotary_dim=64, interleaved=True,
             base=500000.0, scaling="parts", factor=8.0, magnitude=1.2, start=120000,
             name="rotary_wide_step"),
    ]


STEP_BYTES = 1.0e9       # of the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm_step", "norm_step", "drop", "drop", "res", "res_step",
                         "res_step", "rot_step", "rot_step", "append"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op in ("rot_step", "append"):
            d = rng.choice([64, 64, 128, 128, 80, 96, 256])
            kv = _log_int(rng, 1, 32)
            heads = kv * rng.choice([1, 1, 2, 4, 5, 8])
            if heads > 64:
                continue
            scaling = rng.choice(["none", "none", "linear", "parts"])
            tokens = _log_int(rng, 1, 4096)
            capacity = 0
            if op == "append":
                tokens = rng.choice([1, 1, 1, 2, 5, 64, 333])
                capacity = tokens + _log_int(rng, 16, 1024)
            c = _rot(op, _log_int(rng, 1, 64), tokens, heads, d, kv_heads=kv,
                     rotary_dim=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.random() < 0.4,
                     dtype=dtype, base=rng.choice([10000.0, 500000.0]), scaling=scaling,
                     factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                     magnitude=rng.choice([1.0, 1.0, 1.1]), capacity=capacity,
                     start=rng.randint(0, capacity - tokens) if capacity else
                     rng.choice([0, 0, _log_int(rng, 1, 1000000)]))
            cache = 2 * c["batch"] * capacity * kv * d
            if work(c)["bytes"] <= STEP_BYTES and cache <= 1.0e8:
                return c
            continue
        cols = _log_int(rng, 16, 16384) + rng.choice([0, 0, 1, 3])
        if rng.random() < 0.5:
            cols = max(8, cols // 64 * 64 if cols > 64 else cols // 8 * 8)
        cols = min(cols, 16384)
        p = 0.0 if op in ("norm", "norm_step", "res") else rng.choice([0.1, 0.1, 0.25, 0.5])
        if op == "res_step" and rng.random() < 0.2:
            p = 0.0
        c = _rows(op, _log_int(rng, 1, 64), _log_int(rng, 1, 4096), cols, dtype=dtype,
                  weight_dtype=rng.choice(["f32", "bf16"]), p=p, site=rng.randint(0, 65535),
                  lens="full" if op == "drop" else rng.choice(["full", "ragged", "empty"]),
                  residual=rng.random() < 0.5 if op == "drop" else True)
        if work(c)["bytes"] <= STEP_BYTES:
            return c


def _lens(case):
    """Rows of each sequence: padded batches hold lengths from half the
    capacity up; "empty" has one of several sequences without any."""
    B, n = case["batch"], case["tokens"]
    if case["lens"] == "full":
        return [n] * B
    out = [n - (37 * b + 11) % max(1, n // 2) for b in range(B)]
    if case["lens"] == "empty" and B > 1:
        out[B // 2] = 0
    return out


def _starts(case):
    """Position of each sequence's first token."""
    spread = 7 if case["op"] == "append" else 13
    return [max(0, case["start"] - spread * b) for b in range(case["batch"])]


def _dtype(case, key="dtype"):
    return torch.float32 if case[key] == "f32" else torch.bfloat16


def _randn(shape, std, dtype, gen):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _is_rotary(case):
    return case["op"] in ("rot_step", "append")


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, op = _dtype(case), case["op"]
    B, S = case["batch"], case["tokens"]
    if _is_rotary(case):
        nh, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
        # views of one packed projection
        qkv = _randn((B, S, (nh + 2 * kvh) * d), 1.0, dt, gen)
        q, k, v = qkv.split([nh * d, kvh * d, kvh * d], dim=2)
        inp = dict(Q=q.unflatten(2, (nh, d)), K=k.unflatten(2, (kvh, d)))
        if op == "append":
            inp["V"] = v.unflatten(2, (kvh, d))
            shape = (B, case["capacity"], kvh, d)
            inp["K_cache"], inp["V_cache"] = _randn(shape, 1.0, dt, gen), _randn(shape, 1.0, dt, gen)
        else:
            inp["dQ"], inp["dK"] = _randn((B, S, nh, d), 1.0, dt, gen), _randn((B, S, kvh, d), 1.0, dt, gen)
        inp["q_start"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
        return inp
    H = case["cols"]
    if case["packed"]:
        x = _randn((B, 3 * S * H), 1.0, dt, gen)[:, :S * H].unflatten(1, (S, H))
    else:
        x = _randn((B, S, H), 1.0, dt, gen)
    inp = dict(x=x)
    if op in ("res", "res_step") or op == "drop" and case["residual"]:
        # (the residual stream has grown over some layers)
        inp["residual"] = _randn((B, S, H), 2.0, dt, gen)
    if op != "drop":
        wdt = _dtype(case, "weight_dtype")
        inp["weight"] = (1.0 + torch.randn(H, generator=gen, device="cuda") * 0.1).to(wdt)
        inp["bias"] = _randn((H,), 0.1, wdt, gen)
        inp["lens"] = None
        if case["lens"] != "full":
            inp["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    if op in ("norm_step", "res_step", "drop"):
        inp["dy"] = _randn((B, S, H), 1.0, dt, gen)
    if op == "res_step":
        inp["dh"] = _randn((B, S, H), 1.0, dt, gen)
    inp["rng"] = None
    if case["p"] > 0.0:
        # (seed, offset), as a training loop holds them on the device
        inp["rng"] = torch.tensor([0x5DEECE66D1234567 ^ (int(seed) * 0x9E3779B9), 1000003 + int(seed)],
                                  dtype=torch.int64, device="cuda")
    return inp


EPS = 1e-5


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if not own:
        if _is_rotary(case):
            st["freqs"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        return st
    from paper_2410_11720_amd import abft
    op = case["op"]
    shape = (case["batch"], case["tokens"])
    if _is_rotary(case):
        st["rotary"] = abft.Rotary(abft.RotaryConfig(
            *shape, case["heads"], case["head_dim"], kv_heads=case["kv_heads"],
            rotary_dim=case["rotary_dim"], interleaved=case["interleaved"], dtype=case["dtype"],
            base=case["base"], scaling=case["scaling"], factor=case["factor"],
            original_len=case["original_len"], magnitude=case["magnitude"]))
    elif op == "drop":
        st["dropout"] = abft.Dropout(abft.DropoutConfig(*shape, case["cols"], dtype=case["dtype"],
                                                        p=case["p"], site=case["site"]))
    else:
        cfg = abft.NormConfig(*shape, case["cols"], dtype=case["dtype"],
                              weight_dtype=case["weight_dtype"], eps=EPS, dropout=case["p"],
                              site=case["site"])
        kind = abft.LayerNorm if op in ("norm", "norm_step") else abft.ResidualNorm
        st["norm"] = kind(cfg, training=op.endswith("_step"))
    return st


def run(st):
    return _run_own(st) if own else _run_plain(st)


# ---- through the package ------------------------------------------------------

def _run_own(st):
    op = st["case"]["op"]
    if op == "append":
        q = st["rotary"].append(st["Q"], st["K"], st["V"], st["K_cache"], st["V_cache"],
                                q_start=st["q_start"])
        return dict(Q=q, K_cache=st["K_cache"], V_cache=st["V_cache"])
    if op == "rot_step":
        q, k = st["rotary"].forward(st["Q"], st["K"], q_start=st["q_start"])
        dq, dk = st["rotary"].backward(st["dQ"], st["dK"], q_start=st["q_start"])
        return dict(Q=q, K=k, dQ=dq, dK=dk)
    if op == "drop":
        y = st["dropout"].forward(st["x"], st["rng"], residual=st.get("residual"))
        return dict(y=y, dx=st["dropout"].backward(st["dy"], st["rng"]))
    norm, w, b, lens = st["norm"], st["weight"], st["bias"], st["lens"]
    if op in ("norm", "norm_step"):
        y = norm.forward(st["x"], w, b, lens=lens)
        if op == "norm":
            return dict(y=y)
        dx, dw, db = norm.backward(st["dy"], st["x"], w, lens=lens)
        return dict(y=y, dx=dx, dweight=dw, dbias=db)
    h, y = norm.forward(st["x"], st["residual"], w, b, rng=st["rng"], lens=lens)
    if op == "res":
        return dict(h=h, y=y)
    dx, dr, dw, db = norm.backward(st["dy"], h, w, dh=st["dh"], rng=st["rng"], lens=lens)
    return dict(h=h, y=y, dx=dx, dresidual=dr, dweight=dw, dbias=db)


# ---- plain forms ----------------------------------------------------------------

def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    dt = _dtype(case)
    if _is_rotary(case):
        return _rotary_plain(st)
    if op == "drop":
        keep = _keep_plain(case, st["rng"])
        y = _dropped_plain(st["x"].float(), keep, case)
        if "residual" in st:
            y = st["residual"].float() + y
        return dict(y=y.to(dt), dx=_dropped_plain(st["dy"].float(), keep, case).to(dt))
    valid = None
    if st["lens"] is not None:
        i = torch.arange(case["tokens"], device="cuda").view(1, -1, 1)
        valid = i < st["lens"].view(-1, 1, 1)
    only = lambda t: t if valid is None else torch.where(valid, t, torch.zeros_like(t))
    out, keep = {}, None
    if op in ("norm", "norm_step"):
        h = only(st["x"].float())
    else:
        x = st["x"].float()
        if case["p"] > 0.0:
            keep = _keep_plain(case, st["rng"])
            x = _dropped_plain(x, keep, case)
        out["h"] = only(st["residual"].float() + x).to(dt)
        h = out["h"].float()
    w = st["weight"].float()
    centred = h - h.mean(dim=2, keepdim=True)
    r = 1.0 / torch.sqrt((centred * centred).mean(dim=2, keepdim=True) + EPS)
    xh = centred * r
    out["y"] = only(xh * w + st["bias"].float()).to(dt)
    if op in ("norm", "res"):
        return out
    dy = only(st["dy"].float())
    g = dy * w
    g = r * (g - g.mean(dim=2, keepdim=True) - xh * (g * xh).mean(dim=2, keepdim=True))
    if op == "res_step":
        g = only(g + st["dh"].float())
        out["dresidual"] = g.to(dt)
        if keep is not None:
            g = _dropped_plain(g, keep, case)
    out["dx"] = only(g).to(dt)
    out["dweight"] = (dy * xh).sum(dim=(0, 1), dtype=torch.float64).float()
    out["dbias"] = dy.sum(dim=(0, 1), dtype=torch.float64).float()
    return out


def _threshold(case):
    return math.floor(65536 * case["p"] + 0.5)


def _dropped_plain(x, keep, case):
    scale = 65536 / (65536 - _threshold(case))
    return torch.where(keep, x * scale, torch.zeros_like(x))


M32 = 0xFFFFFFFF


def _keep_plain(case, rng):
    """[batch, tokens, cols] truth values: the elements that stay."""
    B, S, H = case["batch"], case["tokens"], case["cols"]
    chunks = (H + 7) // 8
    halves = lambda v: (v & M32, (v >> 32) & M32)
    k0, k1 = halves(rng[0])
    c2, c3 = halves(rng[1])
    c0 = (torch.arange(chunks, device="cuda") + (case["site"] << 13)).view(1, -1)
    c1 = torch.arange(B * S, device="cuda").view(-1, 1)
    for _ in range(10):
        # (products modulo 2^64; the shift's copies of the sign are masked)
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        (l0, h0), (l1, h1) = halves(p0), halves(p1)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=2)
    u = torch.stack([words & 0xFFFF, words >> 16], dim=3).view(B, S, chunks * 8)
    return u[:, :, :H] >= _threshold(case)


def _frequencies(case):
    """Radians a position, of each pair."""
    n, base = case["rotary_dim"], case["base"]
    out = []
    for k in range(n // 2):
        f = base ** (-2.0 * k / n)
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "parts":
            # turns over the length trained on: from 32 up as it is, up to 1 divided
            turns = case["original_len"] * f / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / (32.0 - 1.0)))
            f = f / case["factor"] * (1.0 - keep) + f * keep
        out.append(f)
    return out


def _turn_plain(t, cos, sin, case):
    """One tensor [batch, tokens, heads, head_dim], turned."""
    n = case["rotary_dim"]
    x = t.float()
    if case["interleaved"]:
        a, c = x[..., 0:n:2], x[..., 1:n:2]
        turned = torch.stack([a * cos - c * sin, a * sin + c * cos], dim=4).flatten(3)
    else:
        a, c = x[..., :n // 2], x[..., n // 2:n]
        turned = torch.cat([a * cos - c * sin, a * sin + c * cos], dim=3)
    return torch.cat([turned, x[..., n:]], dim=3).to(t.dtype)


def _rotary_plain(st):
    case = st["case"]
    at = (st["q_start"].view(-1, 1) + torch.arange(case["tokens"], device="cuda")).double()
    angle = at[:, :, None, None] * st["freqs"]
    m = case["magnitude"]
    cos, sin = (torch.cos(angle) * m).float(), (torch.sin(angle) * m).float()
    q, k = _turn_plain(st["Q"], cos, sin, case), _turn_plain(st["K"], cos, sin, case)
    if case["op"] == "append":
        b = torch.arange(case["batch"], device="cuda").view(-1, 1)
        rows = st["q_start"].view(-1, 1).long() + torch.arange(case["tokens"], device="cuda")
        st["K_cache"][b, rows] = k
        st["V_cache"][b, rows] = st["V"]
        return dict(Q=q, K_cache=st["K_cache"], V_cache=st["V_cache"])
    return dict(Q=q, K=k, dQ=_turn_plain(st["dQ"], cos, -sin, case),
                dK=_turn_plain(st["dK"], cos, -sin, case))


# ---- work ------------------------------------------------------------------------

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if _is_rotary(case):
        tokens, d = case["batch"] * case["tokens"], case["head_dim"]
        nh, kvh, rot = case["heads"], case["kv_heads"], case["rotary_dim"]
        if op == "append":
            return dict(bytes=2 * tokens * (nh + 2 * kvh) * d * es, flops=3 * tokens * (nh + kvh) * rot)
        return dict(bytes=4 * tokens * (nh + kvh) * d * es, flops=6 * tokens * (nh + kvh) * rot)
    H = case["cols"]
    n = case["batch"] * case["tokens"] * H
    if op == "drop":
        return dict(bytes=(5 if case["residual"] else 4) * n * es, flops=(3 if case["residual"] else 2) * n)
    # rows behind a sequence's length are written (as zeros), not read
    held = sum(_lens(case)) * H
    wes = 4 if case["weight_dtype"] == "f32" else 2
    params = 2 * H * wes
    read, write, flops = {"norm": (1, 1, 8), "norm_step": (2, 2, 20), "res": (2, 2, 9),
                          "res_step": (4, 4, 24)}[op]
    grads = 8 * H if op.endswith("_step") else 0
    return dict(bytes=(read * held + write * n) * es + params + grads, flops=flops * held)


# ---- from the definition in 64 bits --------------------------------------------------

def _wide(a, b):
    """High and low 32 bits of the product of numbers below 2^32, by their
    16-bit halves (b a plain number)."""
    al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    low = al * bl
    mid = ah * bl + (low >> 16)
    mid2 = al * bh + (mid & 0xFFFF)
    return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_kept(case, rng, first, rows):
    """Kept elements of `rows` rows from `first` on: [rows, cols]."""
    seed, offset = (int(v) % 2 ** 64 for v in rng.tolist())
    H = case["cols"]
    col = torch.arange((H + 7) // 8, device="cuda").repeat(rows, 1)
    x = [col + case["site"] * 8192, torch.zeros_like(col), torch.full_like(col, offset % 2 ** 32),
         torch.full_like(col, offset // 2 ** 32)]
    x[1] += torch.arange(first, first + rows, device="cuda")[:, None]
    for i in range(10):
        key = ((seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)
        hi0, lo0 = _wide(x[0], 0xD2511F53)
        hi1, lo1 = _wide(x[2], 0xCD9E8D57)
        x = [hi1 ^ x[1] ^ key[0], lo1, hi0 ^ x[3] ^ key[1], lo0]
    u = torch.empty((rows, col.shape[1], 8), dtype=torch.int32, device="cuda")
    for i in range(4):
        u[:, :, 2 * i] = x[i] % 65536
        u[:, :, 2 * i + 1] = x[i] // 65536
    return u.view(rows, -1)[:, :H] >= int(case["p"] * 65536 + 0.5)


def _exact_scaled(case, rng, t):
    """Dropout of t [batch, tokens, cols] (64 bits)."""
    if case["p"] == 0.0:
        return t.clone()
    flat = t.reshape(-1, case["cols"])
    out = torch.zeros_like(flat)
    step = max(1, 2 ** 24 // case["cols"])
    factor = 65536.0 / (65536 - int(case["p"] * 65536 + 0.5))
    for at in range(0, flat.shape[0], step):
        part = flat[at:at + step]
        kept = _exact_kept(case, rng, at, part.shape[0])
        out[at:at + step][kept] = part[kept] * factor
    return out.view(t.shape)


def _exact_rotary(case, inp):
    n, sign = case["rotary_dim"], {"Q": 1.0, "K": 1.0, "dQ": -1.0, "dK": -1.0}
    k = torch.arange(n // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(-2.0 * k / n * math.log(case["base"]))
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "parts":
        ramp = ((case["original_len"] * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * (ramp + (1 - ramp) / case["factor"])
    out = {}
    for name, s in sign.items():
        if name not in inp:
            continue
        t = inp[name].double()
        res = t.clone()
        for b, start in enumerate(_starts(case)):
            pos = torch.arange(start, start + case["tokens"], dtype=torch.float64, device="cuda")
            turn = torch.polar(torch.full((case["tokens"], 1, n // 2), case["magnitude"],
                                          dtype=torch.float64, device="cuda"),
                               s * pos[:, None, None] * f)
            if case["interleaved"]:
                z = torch.complex(t[b, :, :, 0:n:2], t[b, :, :, 1:n:2]) * turn
                res[b, :, :, 0:n:2], res[b, :, :, 1:n:2] = z.real, z.imag
            else:
                z = torch.complex(t[b, :, :, :n // 2], t[b, :, :, n // 2:n]) * turn
                res[b, :, :, :n // 2], res[b, :, :, n // 2:n] = z.real, z.imag
        out[name] = res
    if case["op"] != "append":
        return {name: out[name] for name in ("Q", "K", "dQ", "dK")}
    kc, vc = inp["K_cache"].double(), inp["V_cache"].double()
    for b, start in enumerate(_starts(case)):
        kc[b, start:start + case["tokens"]] = out["K"][b]
        vc[b, start:start + case["tokens"]] = inp["V"][b].double()
    return dict(Q=out["Q"], K_cache=kc, V_cache=vc)


def exact(case, seed):
    inp = _inputs(case, seed)
    if _is_rotary(case):
        return _exact_rotary(case, inp)
    op = case["op"]
    if op == "drop":
        y = _exact_scaled(case, inp["rng"], inp["x"].double())
        if "residual" in inp:
            y += inp["residual"].double()
        return dict(y=y, dx=_exact_scaled(case, inp["rng"], inp["dy"].double()))
    out = {}
    h = inp["x"].double()
    if op in ("res", "res_step"):
        out["h"] = _exact_scaled(case, inp["rng"], h) + inp["residual"].double()
        h = out["h"].to(_dtype(case)).double()     # the norm's input is what is stored
    out["y"] = torch.zeros_like(h)
    step = op.endswith("_step")
    if step:
        out["dx"] = torch.zeros_like(h)
        out["dweight"] = torch.zeros(case["cols"], dtype=torch.float64, device="cuda")
        out["dbias"] = torch.zeros_like(out["dweight"])
    w, bias = inp["weight"].double(), inp["bias"].double()
    for b, n in enumerate(_lens(case)):
        if op in ("res", "res_step"):
            out["h"][b, n:] = 0.0
        if n == 0:
            continue
        x = h[b, :n]
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        xh = (x - mean) / sd
        out["y"][b, :n] = xh * w + bias
        if step:
            dy = inp["dy"][b, :n].double()
            out["dbias"] += dy.sum(dim=0)
            out["dweight"] += (dy * xh).sum(dim=0)
            g = dy * w
            # the projection of g off the constant row and off xh, over the deviation
            g = g - (g.sum(dim=1, keepdim=True) + xh * (g * xh).sum(dim=1, keepdim=True)) / case["cols"]
            out["dx"][b, :n] = g / sd
    if op == "res_step":
        for b, n in enumerate(_lens(case)):
            out["dx"][b, :n] += inp["dh"][b, :n].double()
        out["dresidual"] = out["dx"]
        out["dx"] = _exact_scaled(case, inp["rng"], out["dx"])
    order = {"norm": ("y",), "norm_step": ("y", "dx", "dweight", "dbias"), "res": ("h", "y"),
             "res_step": ("h", "y", "dx", "dresidual", "dweight", "dbias")}[op]
    return {name: out[name] for name in order}
