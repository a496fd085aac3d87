"""Attention over keys of another length (cross attention, with an optional
learned relative position bias by buckets), and the global norm and clipping
of gradients, as cases to measure: the calls an encoder-decoder training step
and its decoding make next to the protected layer.

A case's `op`:
  "step"   CrossAttention.forward, then .backward
  "token"  CrossAttention.forward of the last tokens against cached keys
  "clip"   GradientClip.clip of one model's gradients
  "norm"   GradientClip.norm of them

`run` in plain torch (`own` false) or through the package's entry points
(`own` true). Attention, for query i of sequence b and key j:

  s_ij = scale q_i . k_j + table[bucket(j - (start_b + i))]
  allowed: j < len_b, and j <= start_b + i under a causal mask
  o_i = sum_j softmax_j(s_ij) v_j   (0 for a row with no allowed key)
"""
import math

import torch

own = False


# ---- cases ------------------------------------------------------------------

def _att(op, batch, q_len, k_len, heads, head_dim, *, kv_heads=0, dtype="bf16", causal=False,
         lens="full", buckets=0, max_distance=128, name=None):
    c = dict(op=op, batch=batch, q_len=q_len, k_len=k_len, heads=heads,
             kv_heads=kv_heads or heads, head_dim=head_dim, dtype=dtype, causal=causal, lens=lens,
             buckets=buckets, max_distance=max_distance)
    if name:
        c["name"] = name
    return c


def _grads(op, hidden, layers, dtype, name=None):
    c = dict(op=op, hidden=hidden, layers=layers, dtype=dtype, max_norm=1.0)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decoded token against a short encoder output: the smallest call, latency alone
        _att("token", 1, 1, 77, 12, 64, name="token_short"),
        # a batch of decoded tokens against padded encoder states of odd lengths
        _att("token", 32, 1, 1500, 32, 128, lens="ragged", name="token_batch"),
        # decoded tokens over a long self-attention cache, with the decoder's one-sided bias
        _att("token", 48, 1, 4096, 12, 64, causal=True, lens="ragged", buckets=32,
             name="token_bias_cache"),
        # four tokens a sequence at a time, eight shared key heads, a long cache
        _att("token", 4, 4, 8192, 40, 128, kv_heads=8, causal=True, lens="ragged",
             name="tokens_shared_heads"),
        # cross attention of a training step: targets of 512 over padded sources of 1000
        _att("step", 8, 512, 1000, 12, 64, lens="ragged", name="cross_step"),
        # the same of a wide layer, key heads shared by four: the largest
        _att("step", 4, 2048, 1024, 32, 128, kv_heads=8, name="cross_step_wide"),
        # encoder self attention with a two-sided bias over padded sources
        _att("step", 8, 512, 512, 12, 64, lens="ragged", buckets=32, name="encoder_bias_step"),
        # decoder self attention, causal, with a one-sided bias
        _att("step", 8, 1024, 1024, 12, 64, causal=True, buckets=32, name="decoder_bias_step"),
        # full precision, odd lengths
        _att("step", 2, 200, 333, 12, 64, dtype="f32", lens="ragged", buckets=32,
             name="cross_step_f32"),
        # one small layer: a few tensors of 64 to 12288 elements
        _grads("clip", 64, 1, "f32", name="clip_small"),
        # the gradients of twelve GPT-2 attention layers
        _grads("clip", 768, 12, "f32", name="clip_model"),
        # the norm alone, two attention layers of the large decoder, gradients in bf16
        _grads("norm", 4096, 2, "bf16", name="norm_wide"),
    ]


STEP_FLOPS = 4.0e11      # of the largest listed step
STEP_FLOPS_F32 = 1.0e10
TOKEN_BYTES = 6.0e8
GRAD_ELEMENTS = 4.0e8


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["step", "step", "step", "step", "f32", "token", "token", "token",
                           "clip", "norm"])
        if kind in ("clip", "norm"):
            c = _grads(kind, 8 * _log_int(rng, 4, 512) + rng.choice([0, 0, 1, 3]),
                       _log_int(rng, 1, 24), rng.choice(["f32", "f32", "bf16"]))
            if sum(_sizes(c)) <= GRAD_ELEMENTS:
                return c
            continue
        d = rng.choice([64, 64, 128])
        kv = _log_int(rng, 1, 32)
        heads = kv * rng.choice([1, 1, 2, 4, 5, 8])
        causal = rng.random() < 0.4
        buckets = rng.choice([0, 0, 8, 32, 32, 64])
        lens = rng.choice(["full", "ragged", "ragged", "empty"])
        if heads > 64:
            continue
        if kind == "token":
            q_len = rng.choice([1, 1, 1, 2, 4, 7, 8])
            c = _att("token", _log_int(rng, 1, 64), q_len, _log_int(rng, 16, 16384), heads, d,
                     kv_heads=kv, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
                     causal=causal, lens=lens, buckets=buckets,
                     max_distance=rng.choice([64, 128, 128, 256]))
            if work(c)["bytes"] <= TOKEN_BYTES:
                return c
            continue
        q_len = _log_int(rng, 1, 2500)
        k_len = q_len if causal else _log_int(rng, 1, 2500)
        dtype = "f32" if kind == "f32" else "bf16"
        c = _att("step", _log_int(rng, 1, 16), q_len, k_len, heads, d, kv_heads=kv, dtype=dtype,
                 causal=causal, lens=lens, buckets=buckets,
                 max_distance=rng.choice([64, 128, 128, 256]))
        if work(c)["flops"] > (STEP_FLOPS_F32 if dtype == "f32" else STEP_FLOPS):
            continue
        if c["batch"] * heads * q_len * k_len > 4.0e8:  # the plain form's scores
            continue
        return c


def _lens(case):
    """Keys of each sequence: padded batches hold lengths from half the
    capacity up; "empty" has one sequence without any."""
    B, n = case["batch"], case["k_len"]
    if case["lens"] == "full":
        return [n] * B
    out = [n - (37 * b + 11) % max(1, n // 2) for b in range(B)]
    if case["lens"] == "empty":
        out[B // 2] = 0
    return out


def _starts(case):
    """Position of each sequence's first query among its keys: decoded
    tokens are the last ones of their sequence."""
    if case["op"] == "token" and case["causal"]:
        return [n - case["q_len"] for n in _lens(case)]
    return None


def _sizes(case):
    """Elements of each gradient: per attention layer the projections, their
    biases, a norm's gain and offset."""
    h = case["hidden"]
    return [3 * h * h, h * h, 3 * h, h, h, h] * case["layers"]


def _flat(case, dtype):
    """One buffer for the clipped gradients, each at a multiple of 64
    elements (zeros between them), and its views."""
    starts, n = [], 0
    for size in _sizes(case):
        starts.append(n)
        n += (size + 63) // 64 * 64
    flat = torch.zeros((n,), dtype=dtype, device="cuda")
    return flat, [flat[at:at + size] for at, size in zip(starts, _sizes(case))]


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _randn(shape, std, dtype, gen):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _dtype(case)
    if case["op"] in ("clip", "norm"):
        return dict(grads=[_randn((n,), 0.01, dt, gen) for n in _sizes(case)])
    B, Sq, Sk = case["batch"], case["q_len"], case["k_len"]
    nh, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
    # views as the projections leave them: queries [B, Sq, nh, d]; keys and
    # values the two halves of one packed tensor
    Q = _randn((B, Sq, nh, d), 1.0, dt, gen)
    KV = _randn((B, Sk, 2, kvh, d), 1.0, dt, gen)
    inp = dict(Q=Q, K=KV[:, :, 0], V=KV[:, :, 1], bias=None, k_lens=None, q_start=None)
    if case["op"] == "step":
        inp["dO"] = _randn((B, Sq, nh, d), 1.0, dt, gen)
    if case["buckets"]:
        inp["bias"] = _randn((case["buckets"], nh), 1.0, torch.float32, gen)
    if case["lens"] != "full":
        inp["k_lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    if _starts(case) is not None:
        inp["q_start"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda")
    return inp


def prepare(case, seed):
    st = dict(case=case, **_inputs(case, seed))
    if case["op"] in ("clip", "norm"):
        if case["op"] == "clip":
            st["flat"], st["out"] = _flat(case, _dtype(case))
        if own:
            from paper_2410_11720_amd import abft
            st["clipper"] = abft.GradientClip(st["grads"])
        return st
    if own:
        from paper_2410_11720_amd import abft
        st["attention"] = abft.CrossAttention(abft.CrossConfig(
            case["batch"], case["q_len"], case["k_len"], case["heads"], case["head_dim"],
            kv_heads=case["kv_heads"], dtype=case["dtype"], causal=case["causal"],
            buckets=case["buckets"], max_distance=case["max_distance"],
            bidirectional=not case["causal"]))
    return st


def run(st):
    op = st["case"]["op"]
    if op in ("clip", "norm"):
        return _run_grads_own(st) if own else _run_grads_plain(st)
    return _run_attention_own(st) if own else _run_attention_plain(st)


# ---- through the package ------------------------------------------------------

def _run_grads_own(st):
    clipper = st["clipper"]
    if st["case"]["op"] == "norm":
        clipper.norm(st["grads"])
        return dict(norm=clipper.stats.norm, nonfinite=clipper.stats.nonfinite)
    clipper.clip(st["grads"], st["case"]["max_norm"], out=st["out"])
    return dict(out=st["flat"], norm=clipper.stats.norm, coef=clipper.stats.coef,
                nonfinite=clipper.stats.nonfinite)


def _run_attention_own(st):
    att = st["attention"]
    keys = dict(bias=st["bias"], k_lens=st["k_lens"], q_start=st["q_start"])
    O = att.forward(st["Q"], st["K"], st["V"], **keys)
    if st["case"]["op"] == "token":
        return dict(O=O)
    dQ, dK, dV, dbias = att.backward(st["dO"], st["Q"], st["K"], st["V"], O, **keys)
    return dict(O=O, dQ=dQ, dK=dK, dV=dV, dbias=dbias)


# ---- plain forms ----------------------------------------------------------------

def _run_grads_plain(st):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    nonfinite = torch.zeros((), dtype=torch.int64, device="cuda")
    for g in st["grads"]:
        g = g.float()
        total += (g * g).sum(dtype=torch.float64)
        nonfinite += (~torch.isfinite(g)).sum()
    norm = total.sqrt().float()
    if st["case"]["op"] == "norm":
        return dict(norm=norm, nonfinite=nonfinite)
    coef = (st["case"]["max_norm"] / norm.double()).clamp(max=1.0).float()
    for g, o in zip(st["grads"], st["out"]):
        o.copy_(g.float() * coef)
    return dict(out=st["flat"], norm=norm, coef=coef, nonfinite=nonfinite)


def _relative_plain(case, start):
    """j - (start + i) for all pairs: [B or 1, Sq, Sk]."""
    q = torch.arange(case["q_len"], device="cuda").view(1, -1, 1)
    k = torch.arange(case["k_len"], device="cuda").view(1, 1, -1)
    return k - q if start is None else k - (q + start.long().view(-1, 1, 1))


def _bucket_plain(rel, case):
    """Bucket of a relative position: half of a side's buckets one per
    distance, the others by the logarithm of the distance up to
    max_distance; a two-sided table's second half for keys ahead."""
    n_buckets = case["buckets"]
    base = torch.zeros_like(rel)
    if case["causal"]:
        n = (-rel).clamp(min=0)
    else:
        n_buckets //= 2
        base = (rel > 0).long() * n_buckets
        n = rel.abs()
    exact = n_buckets // 2
    far = (torch.log(n.clamp(min=1).double() / exact) / math.log(case["max_distance"] / exact)
           * (n_buckets - exact))
    # (a distance on a border, n = exact (max / exact)^(t / far buckets),
    # belongs to bucket t; the other ones lie further from it than 1e-9)
    far = (exact + torch.floor(far + 1e-9).long()).clamp(max=n_buckets - 1)
    return base + torch.where(n < exact, n, far)


def _allowed_plain(st, case):
    """[B or 1, 1, Sq, Sk] truth values."""
    j = torch.arange(case["k_len"], device="cuda").view(1, 1, 1, -1)
    ok = torch.ones((1, 1, case["q_len"], case["k_len"]), dtype=torch.bool, device="cuda")
    if st["k_lens"] is not None:
        ok = ok & (j < st["k_lens"].view(-1, 1, 1, 1))
    if case["causal"]:
        ok = ok & (_relative_plain(case, st["q_start"]).unsqueeze(1) <= 0)
    return ok


def _run_attention_plain(st):
    case = st["case"]
    dt = _dtype(case)
    group = case["heads"] // case["kv_heads"]
    scale = 1.0 / math.sqrt(case["head_dim"])
    q = st["Q"].float().transpose(1, 2).contiguous()
    k = st["K"].float().transpose(1, 2).repeat_interleave(group, dim=1)
    v = st["V"].float().transpose(1, 2).repeat_interleave(group, dim=1)
    ok = _allowed_plain(st, case)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    if case["buckets"]:
        bucket = _bucket_plain(_relative_plain(case, st["q_start"]), case)
        s = s + st["bias"][bucket].permute(0, 3, 1, 2)
    s = s.masked_fill(~ok, -math.inf)
    top = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, v)
    out = o.transpose(1, 2).to(dt).contiguous()
    if case["op"] == "token":
        return dict(O=out)
    do = st["dO"].float().transpose(1, 2).contiguous()
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(dim=3, keepdim=True))
    B, kvh, Sk, d = case["batch"], case["kv_heads"], case["k_len"], case["head_dim"]
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * scale
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    dk = dk.view(B, kvh, group, Sk, d).sum(dim=2)
    dv = dv.view(B, kvh, group, Sk, d).sum(dim=2)
    dbias = None
    if case["buckets"]:
        flat = ds.sum(dim=0, dtype=torch.float64).view(case["heads"], -1)
        which = bucket.view(1, -1)
        dbias = torch.stack([(flat * (which == t)).sum(dim=1) for t in range(case["buckets"])])
        dbias = dbias.float()
    return dict(O=out, dQ=dq.transpose(1, 2).to(dt).contiguous(),
                dK=dk.transpose(1, 2).to(dt).contiguous(),
                dV=dv.transpose(1, 2).to(dt).contiguous(), dbias=dbias)


# ---- work ------------------------------------------------------------------------

def _pairs(case):
    """Allowed (query, key) pairs over the batch, of one head."""
    total = 0
    starts = _starts(case) or [0] * case["batch"]
    for n, start in zip(_lens(case), starts):
        if not case["causal"]:
            total += n * case["q_len"]
            continue
        for i in range(case["q_len"]):
            total += max(0, min(n, start + i + 1))
    return total


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("clip", "norm"):
        n = sum(_sizes(case))
        return dict(bytes=n * es * (2 if case["op"] == "clip" else 1),
                    flops=n * (3 if case["op"] == "clip" else 2))
    nh, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
    q = case["batch"] * case["q_len"] * nh * d * es
    kv = 2 * sum(_lens(case)) * kvh * d * es
    bias = 4 * case["buckets"] * nh
    fwd = 4 * d * nh * _pairs(case)
    if case["op"] == "token":
        return dict(bytes=2 * q + kv + bias, flops=fwd)
    # two products forward and four backward; the gradients of every key row,
    # also behind a sequence's length, are written
    grads = 2 * case["batch"] * case["k_len"] * kvh * d * es
    return dict(bytes=4 * q + kv + grads + 2 * bias, flops=3 * fwd)


# ---- from the definition in 64 bits --------------------------------------------------

def _exact_buckets(case):
    """Bucket of every distance 0..max_distance on one side, in whole
    numbers: distance n is in log bucket t or above if
    (n / e)^f >= (max / e)^t, with e exact and f log buckets."""
    nb = case["buckets"] if case["causal"] else case["buckets"] // 2
    e, top = nb // 2, case["max_distance"]
    f = nb - e
    out = []
    for n in range(top + 1):
        if n < e:
            out.append(n)
            continue
        t = 0
        while t < f - 1 and n ** f >= e ** (f - (t + 1)) * top ** (t + 1):
            t += 1
        out.append(e + t)
    return nb, out


def _exact_grads(case, inp):
    total = 0.0
    bad = 0
    for g in inp["grads"]:
        g = g.double()
        bad += int((~torch.isfinite(g)).sum())
        total += float(torch.dot(g, g))
    norm = math.sqrt(total)
    one = lambda x: torch.tensor(x, dtype=torch.float64, device="cuda")
    if case["op"] == "norm":
        return dict(norm=one(norm), nonfinite=torch.tensor(bad, device="cuda"))
    coef = min(1.0, case["max_norm"] / norm)
    flat, views = _flat(case, torch.float64)
    for g, o in zip(inp["grads"], views):
        o.copy_(g.double() * coef)
    return dict(out=flat, norm=one(norm), coef=one(coef),
                nonfinite=torch.tensor(bad, device="cuda"))


def exact(case, seed):
    inp = _inputs(case, seed)
    if case["op"] in ("clip", "norm"):
        return _exact_grads(case, inp)
    B, Sq, Sk = case["batch"], case["q_len"], case["k_len"]
    nh, kvh, d = case["heads"], case["kv_heads"], case["head_dim"]
    group, scale = nh // kvh, d ** -0.5
    step = case["op"] == "step"
    lens, starts = _lens(case), _starts(case) or [0] * B
    f64 = dict(dtype=torch.float64, device="cuda")
    O = torch.zeros((B, Sq, nh, d), **f64)
    dQ, dK, dV = torch.zeros_like(O), torch.zeros((B, Sk, kvh, d), **f64), torch.zeros((B, Sk, kvh, d), **f64)
    dbias = torch.zeros((case["buckets"], nh), **f64) if case["buckets"] else None
    side = None
    if case["buckets"]:
        half, side = _exact_buckets(case)
        side = torch.tensor(side, device="cuda")
    for b in range(B):
        n = lens[b]
        if n == 0:
            continue
        pos = torch.arange(starts[b], starts[b] + Sq, device="cuda")
        rel = torch.arange(n, device="cuda")[None, :] - pos[:, None]
        hidden = rel > 0 if case["causal"] else torch.zeros_like(rel, dtype=torch.bool)
        if case["buckets"]:
            dist = torch.where(rel > 0, 0, -rel) if case["causal"] else rel.abs()
            which = side[dist.clamp(max=case["max_distance"])]
            if not case["causal"]:
                which = which + half * (rel > 0)
        for h in range(nh):
            q = inp["Q"][b, :, h].double()
            k, v = inp["K"][b, :n, h // group].double(), inp["V"][b, :n, h // group].double()
            s = (q @ k.T) * scale
            if case["buckets"]:
                s += inp["bias"][:, h].double()[which]
            s[hidden] = -math.inf
            seen = ~hidden.all(dim=1)
            p = torch.zeros_like(s)
            p[seen] = torch.softmax(s[seen], dim=1)
            O[b, :, h] = p @ v
            if not step:
                continue
            g = inp["dO"][b, :, h].double()
            dp = g @ v.T
            ds = p * (dp - (p * dp).sum(dim=1, keepdim=True))
            dQ[b, :, h] = ds @ k * scale
            dK[b, :n, h // group] += ds.T @ q * scale
            dV[b, :n, h // group] += p.T @ g
            if case["buckets"]:
                dbias[:, h] += torch.bincount(which.reshape(-1), weights=ds.reshape(-1),
                                              minlength=case["buckets"])
    return dict(O=O, dQ=dQ, dK=dK, dV=dV, dbias=dbias) if step else dict(O=O)
