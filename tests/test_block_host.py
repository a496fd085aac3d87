"""What the classes of layer norm, dropout and rotary positions do on the host around
their C calls, on CPU tensors: records of a forward, references, arguments. The
library's calls are replaced by one that notes what it is given."""
import sys

import pytest
import torch

from paper_2410_11720_amd import abft


class Host:
    """Stands for the device: CPU tensors are on it."""
    index = -1

    def __eq__(self, other):
        return other == torch.device("cpu")

    def __str__(self):
        return "cpu"


@pytest.fixture
def calls(monkeypatch):
    """(function, arguments) of each call of the library."""
    made = []
    monkeypatch.setattr(abft, "_call", lambda fn, device, *args: made.append((fn, args)) or 0)
    return made


def _host(kind, cfg, **kw):
    op = kind(cfg, device="cpu", **kw)
    op.device = Host()
    return op


def _rows(n=1, shape=(2, 3, 40), dtype=torch.bfloat16):
    out = [torch.zeros(shape, dtype=dtype) for _ in range(n)]
    return out if n > 1 else out[0]


def _norm(kind=abft.LayerNorm, batch=2, **kw):
    return _host(kind, abft.NormConfig(batch, 3, 40, **kw))


def test_a_gradient_on_the_rows_leaves_no_record(calls):
    """dx on x (on h): a further backward would read the gradient as rows."""
    x, dy, other = _rows(3)
    op = _norm()
    op.forward(x)
    op.backward(dy, x, dx=other)
    op.backward(dy, x, dx=dy)
    assert len(calls) == 3
    assert op.backward(dy, x, dx=x)[0] is x
    with pytest.raises(abft.AbftError):
        op.backward(dy, x)
    saved = abft.NormSaved(op.cfg, "cpu")
    op.forward(x, saved=saved)
    op.backward(dy, x, dx=x, saved=saved)
    with pytest.raises(abft.AbftError):
        op.backward(dy, x, saved=saved)
    op.forward(x)
    op.backward(dy, x)

    for name in ("dx", "dresidual"):
        op = _norm(abft.ResidualNorm, dropout=0.5)
        rng = torch.zeros(2, dtype=torch.int64)
        h, _ = op.forward(x, other, rng=rng)
        op.backward(dy, h, rng=rng)
        op.backward(dy, h, rng=rng, **{name: h})
        with pytest.raises(abft.AbftError):
            op.backward(dy, h, rng=rng)


def test_rows_that_took_the_place_of_others(calls):
    """The record is of a tensor's memory and layout: not of what is at its address once
    it is gone, nor of another view from there."""
    import numpy as np
    memory = np.zeros(4000, dtype=np.float32)
    tensor = lambda: torch.from_numpy(memory)[:240].view(2, 3, 40)   # memory given out again
    dy = torch.zeros(2, 3, 40)
    op = _norm(dtype="f32")
    x = tensor()
    op.forward(x)
    op.backward(dy, x)
    op.backward(dy, x.detach())
    op.backward(dy, x.view(6, 40).view(2, 3, 40))
    saved = abft.NormSaved(op.cfg, "cpu")
    op.forward(x, saved=saved)
    op.forward(x)
    with pytest.raises(abft.AbftError):
        op.backward(dy, x.as_strided((2, 3, 40), (120, 80, 1)))
    del x
    x = tensor()
    with pytest.raises(abft.AbftError):
        op.backward(dy, x)
    op.backward(dy, x, saved=saved)        # (the caller's to know)
    view = x.view(6, 40).view(2, 3, 40)
    op.forward(view)
    del view                               # its memory lives on
    op.backward(dy, x)

    op = _norm(abft.ResidualNorm, dtype="f32")
    h = tensor()
    op.forward(x, dy, h=h, y=torch.zeros(2, 3, 40))
    op.backward(dy, h)
    del h
    with pytest.raises(abft.AbftError):
        op.backward(dy, tensor())


@pytest.mark.parametrize("p", [0.0, 0.5])
def test_one_tensor_for_both_gradients(monkeypatch, p):
    """With dropout the call gets both, and refuses them."""
    given = []

    def call(fn, device, *args):
        given.append(args)
        return 0 if len(given) == 1 else -1
    monkeypatch.setattr(abft, "_call", call)
    x, dy, other = _rows(3)
    op = _norm(abft.ResidualNorm, dropout=p)
    rng = torch.zeros(2, dtype=torch.int64)
    h, _ = op.forward(x, other, rng=rng)
    with pytest.raises(abft.AbftError):
        op.backward(dy, h, rng=rng, dx=x, dresidual=x)
    dx, dresidual = given[1][8:10]
    assert dx is not None and (dresidual is not None) == (p > 0)


@pytest.mark.parametrize("kind", [abft.LayerNorm, abft.ResidualNorm])
def test_no_rows_have_a_backward(calls, kind):
    """Tensors without elements all have the address 0: none is on another."""
    op = _norm(kind, batch=0)
    x, dy, other = _rows(3, shape=(0, 3, 40))
    first = (x,) if kind is abft.LayerNorm else (x, other)
    with pytest.raises(abft.AbftError):
        op.backward(dy, x)
    op.forward(*first)
    for kw in ({}, dict(dx=other), dict(dx=x)):
        op.backward(dy, x, **kw)
    op.forward(*first, y=x)
    op.backward(dy, x)
    saved = abft.NormSaved(op.cfg, "cpu")
    op.forward(*first, y=x, saved=saved)
    op.backward(dy, x, dx=x, saved=saved)
    op.backward(dy, x, saved=saved)
    op.backward(dy, x)
    assert len(calls) == 10


def test_results_with_another_record_on_the_rows(calls):
    """The object's own record ends too if a call with another one writes on its rows."""
    x, dy, other = _rows(3)
    op = _norm()
    for write in (lambda s: op.backward(dy, x, dx=x, saved=s), lambda s: op.forward(other, y=x, saved=s),
                  lambda s: op.forward(x, y=x, saved=s)):
        saved = abft.NormSaved(op.cfg, "cpu")
        op.forward(x, saved=saved)
        op.forward(x)
        op.forward(x, y=other, saved=saved)
        op.backward(dy, x)
        write(saved)
        with pytest.raises(abft.AbftError):
            op.backward(dy, x)
    op = _norm(abft.ResidualNorm)
    for name in ("h", "y"):
        saved = abft.NormSaved(op.cfg, "cpu")
        h, _ = op.forward(x, other)
        op.backward(dy, h)
        op.forward(x, other, saved=saved, **{name: h})
        with pytest.raises(abft.AbftError):
            op.backward(dy, h)


FAR = 2 ** 32


@pytest.mark.parametrize("kind,kw", [
    (abft.NormConfig, dict(batch=FAR + 2)), (abft.NormConfig, dict(tokens=FAR + 3)),
    (abft.NormConfig, dict(cols=FAR + 40)), (abft.NormConfig, dict(site=FAR)),
    (abft.NormConfig, dict(site=-1)), (abft.NormConfig, dict(tokens=2 ** 31)),
    (abft.DropoutConfig, dict(batch=FAR + 2)), (abft.DropoutConfig, dict(tokens=FAR + 3)),
    (abft.DropoutConfig, dict(cols=FAR + 40)), (abft.DropoutConfig, dict(site=FAR + 1)),
    (abft.RotaryConfig, dict(batch=FAR + 2)), (abft.RotaryConfig, dict(tokens=FAR + 3)),
    (abft.RotaryConfig, dict(heads=FAR + 4)), (abft.RotaryConfig, dict(kv_heads=FAR + 4)),
    (abft.RotaryConfig, dict(head_dim=FAR + 16)), (abft.RotaryConfig, dict(rotary_dim=FAR + 16))])
def test_sizes_past_their_fields(kind, kw):
    """Refused, not cut to their low 32 bits (a tensor of 2^32 + 3 rows would have three
    of them normalised, site 2^32 the draws of site 0)."""
    base = dict(batch=2, tokens=3)
    base.update(dict(heads=4, head_dim=16) if kind is abft.RotaryConfig else dict(cols=40))
    kind(**base).to_c()
    with pytest.raises(abft.AbftError):
        kind(**{**base, **kw}).to_c()


def test_places_past_their_fields():
    assert abft.attn_dropout_draw(1, 2, 3, FAR - 1, 5) >= 0
    for site, row, col in ((FAR, 0, 0), (-1, 0, 0), (0, FAR, 0), (0, -1, 0), (0, 0, FAR), (0, 0, -8)):
        with pytest.raises(abft.AbftError):
            abft.attn_dropout_draw(1, 2, site, row, col)
    with pytest.raises(abft.AbftError):
        abft.attn_rotary_frequencies(FAR + 4)


def test_a_cache_past_its_field(calls):
    """A capacity of 2^32 + 4 rows is not one of four."""
    rot = _host(abft.Rotary, abft.RotaryConfig(1, 1, 1, 2))
    q = _rows(shape=(1, 1, 1, 2))
    cache = q.expand(1, FAR + 4, 1, 2)
    with pytest.raises(abft.AbftError):
        rot.append(q, q, q, cache, cache)
    rot.append(q, q, q, cache[:, :9], cache[:, :9])
    assert len(calls) == 1


def test_tensors_are_held_until_the_launch(monkeypatch):
    """From Python 3.11 on a method's names are all that holds a temporary that was
    passed to it: each still names its tensor when the library is called, so that no
    allocation in between gets its memory."""
    seen = []

    def call(fn, device, *args):
        f = sys._getframe(1)
        while f.f_code.co_name not in ("forward", "backward", "append"):
            f = f.f_back
        seen.append(dict(f.f_locals))
        return 0
    monkeypatch.setattr(abft, "_call", call)
    rng = torch.zeros(2, dtype=torch.int64)
    w, lens = torch.ones(40), torch.ones(2, dtype=torch.int32)

    def check(method, **given):
        method(**given)
        for name, t in given.items():
            assert t is None or seen[-1][name] is t, (method, name)
    x, r, dy, a, b = _rows(5)
    norm = _norm()
    for y in (None, a):
        check(norm.forward, x=x, weight=w, bias=w, lens=lens, y=y)
        sums = {} if y is None else dict(dweight=w, dbias=w)
        check(norm.backward, dy=dy, x=x, weight=w, lens=lens, dx=y, **sums)
    end = _norm(abft.ResidualNorm, dropout=0.5)
    check(end.forward, x=x, residual=r, weight=w, bias=w, rng=rng, lens=lens)
    check(end.forward, x=x, residual=r, weight=w, bias=w, rng=rng, lens=lens, h=a, y=b)
    check(end.backward, dy=dy, h=a, weight=w, dh=r, rng=rng, lens=lens)
    check(end.backward, dy=dy, h=a, weight=w, dh=r, rng=rng, lens=lens, dx=x, dresidual=b)
    drop = _host(abft.Dropout, abft.DropoutConfig(2, 3, 40))
    check(drop.forward, x=x, rng=rng, residual=r)
    check(drop.forward, x=x, rng=rng, residual=r, y=a)
    check(drop.backward, dy=dy, rng=rng)
    rot = _host(abft.Rotary, abft.RotaryConfig(2, 3, 4, 10))
    q, k, v, o, p = (t.view(2, 3, 4, 10) for t in (x, r, dy, a, b))
    for name in ("", "d"):
        method = rot.backward if name else rot.forward
        check(method, **{name + "Q": q, name + "K": k}, q_start=lens)
        check(method, q_start=lens,
              **{name + "Q": q, name + "K": k, name + "Q_out": o, name + "K_out": p})
    check(rot.append, Q=q, K=k, V=v, K_cache=o, V_cache=p, q_start=lens)
    check(rot.append, Q=q, K=k, V=v, K_cache=o, V_cache=p, q_start=lens, Q_out=q)


def test_results_beside_overlapping_rows(calls):
    """Rows that move on by one element (windows of one buffer): torch.empty_like of them
    has no contiguous columns; the results have."""
    flat = torch.zeros(4000, dtype=torch.bfloat16)
    x = flat.as_strided((2, 3, 40), (100, 1, 1))
    y = flat.as_strided((2, 3, 40), (1, 100, 1))
    dy = _rows()
    rng = torch.zeros(2, dtype=torch.int64)
    assert torch.empty_like(x).stride(2) != 1 and torch.empty_like(y).stride(2) != 1
    out = []
    for t in (x, y):
        norm, end = _norm(), _norm(abft.ResidualNorm, dropout=0.5)
        out += [norm.forward(t), norm.backward(t, t)[0]]
        h, n = end.forward(t, dy, rng=rng)
        out += [h, n, *end.backward(t, h, rng=rng)[:2], *end.backward(t, h, rng=rng, dx=dy)[:2]]
        out += [end.forward(t, dy, rng=rng, h=dy)[1], end.forward(t, dy, rng=rng, y=dy)[0]]
        drop = _host(abft.Dropout, abft.DropoutConfig(2, 3, 40))
        out += [drop.forward(t, rng), drop.backward(t, rng)]
    rot = _host(abft.Rotary, abft.RotaryConfig(2, 3, 2, 40))
    q = flat.as_strided((2, 3, 2, 40), (100, 40, 1, 1))
    k = torch.zeros((2, 3, 2, 40), dtype=torch.bfloat16)
    assert torch.empty_like(q).stride(3) != 1
    out += [*rot.forward(q, k), *rot.forward(k, q), *rot.backward(q, k), rot.forward(q, k, K_out=k)[0],
            rot.forward(k, q, Q_out=k)[1], rot.append(q, k, k, k, k)]
    for t in out:
        st = t.stride()
        assert st[-1] == 1 and t.shape in (x.shape, q.shape) and t.dtype == x.dtype
        assert t.is_contiguous() or sorted(st)[1] >= 40


def _valid():
    """A call of each method with tensors as they have to be: name -> (method, arguments)."""
    x, r, dy, o, p = _rows(5)
    rng, w = torch.zeros(2, dtype=torch.int64), torch.ones(40)
    lens = torch.ones(2, dtype=torch.int32)
    norm, end = _norm(), _norm(abft.ResidualNorm, dropout=0.5)
    drop = _host(abft.Dropout, abft.DropoutConfig(2, 3, 40))
    rot = _host(abft.Rotary, abft.RotaryConfig(2, 3, 4, 10, kv_heads=2))
    norm.forward(x)
    h, _ = end.forward(x, r, rng=rng)
    q, k = torch.zeros((2, 3, 4, 10)).bfloat16(), torch.zeros((2, 3, 2, 10)).bfloat16()
    cache = torch.zeros((2, 9, 2, 10)).bfloat16()
    return {
        "norm": (norm.forward, dict(x=x, weight=w, bias=w, lens=lens, y=o)),
        "norm back": (norm.backward, dict(dy=dy, x=x, weight=w, lens=lens, dx=o, dweight=w, dbias=w)),
        "end": (end.forward, dict(x=x, residual=r, weight=w, bias=w, rng=rng, lens=lens, h=o, y=p)),
        "end back": (end.backward, dict(dy=dy, h=h, weight=w, dh=r, rng=rng, lens=lens, dx=o,
                                        dresidual=p, dweight=w, dbias=w)),
        "drop": (drop.forward, dict(x=x, rng=rng, residual=r, y=o)),
        "drop back": (drop.backward, dict(dy=dy, rng=rng, dx=o)),
        "turn": (rot.forward, dict(Q=q, K=k, q_start=lens, Q_out=q, K_out=k)),
        "turn back": (rot.backward, dict(dQ=q, dK=k, q_start=lens, dQ_out=q, dK_out=k)),
        "append": (rot.append, dict(Q=q, K=k, V=k, K_cache=cache, V_cache=cache, q_start=lens, Q_out=q)),
    }


VECTORS = ("weight", "bias", "lens", "rng", "q_start", "dweight", "dbias")
OPTIONAL = VECTORS + ("y", "dx", "dresidual", "dh", "Q_out", "K_out", "dQ_out", "dK_out")


@pytest.mark.parametrize("name", ["norm", "norm back", "end", "end back", "drop", "drop back", "turn",
                                  "turn back", "append"])
def test_each_argument_is_looked_at(calls, name):
    """The call passes as it stands and without what is optional; each tensor of another
    type, shape or layout is refused, before the library is called, by its name, and tensors
    of another device are."""
    method, given = _valid()[name]
    made = len(calls)
    method(**given)
    for arg in given:
        needed = name.startswith(("end", "drop")) and arg == "rng"
        if arg in OPTIONAL and not needed:
            method(**{k: v for k, v in given.items() if k != arg})
    passed = len(calls)
    assert passed > made
    for arg, t in given.items():
        wide = torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype)
        bad = [t.half() if t.dtype != torch.int64 else t.int(), t[..., :-1], t[None], wide[..., ::2]]
        if arg in VECTORS:
            bad.append(torch.zeros(t.numel() + 1, dtype=t.dtype))
        elif "cache" not in arg:
            bad.append(torch.cat([t, t], dim=1))
        else:
            bad.append(torch.cat([t, t], dim=0))
        for other in bad:
            with pytest.raises(abft.AbftError) as e:
                method(**{**given, arg: other})
            said = str(e.value)
            assert arg in said or "not those of the last forward" in said, (arg, other.shape)
    method.__self__.device.index = 0
    with pytest.raises(abft.AbftError):
        method(**given)
    assert len(calls) == passed
