"""What a CrossAttention forward leaves for its backward: taken only with the O
it belongs to, and kept apart where forwards come in between."""
import pytest
import torch

from paper_2410_11720_amd import abft

C = abft.CrossConfig


def _inputs(cfg, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = cfg.torch_dtype
    q, g = (torch.randn((cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim), generator=gen,
                        device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn((cfg.batch, cfg.k_len, cfg.heads, cfg.head_dim), generator=gen,
                        device="cuda").to(dt) for _ in range(2))
    return q, k, v, g


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_forwards_in_between(dtype):
    """Two layers through one object, then their backwards in turn."""
    cfg = C(2, 50, 80, 2, 64, dtype=dtype)
    one, two = _inputs(cfg, 1), _inputs(cfg, 2)
    want = []
    for q, k, v, g in (one, two):
        att = abft.CrossAttention(cfg)
        o = att.forward(q, k, v)
        want.append(att.backward(g, q, k, v, o)[:3])
    att = abft.CrossAttention(cfg)
    # one's statistics are gone after two's forward: refused, not mixed
    o1 = att.forward(*one[:3])
    o2 = att.forward(*two[:3])
    with pytest.raises(abft.AbftError):
        att.backward(one[3], *one[:3], o1)
    got = att.backward(two[3], *two[:3], o2)[:3]
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    # a record each
    saved = [att.new_saved(), att.new_saved()]
    o1 = att.forward(*one[:3], saved=saved[0])
    o2 = att.forward(*two[:3], saved=saved[1])
    att.forward(*two[:3])
    for (q, k, v, g), o, s, w in ((one, o1, saved[0], want[0]), (two, o2, saved[1], want[1])):
        # (a copy of O will do: the caller knows that it belongs to the record)
        got = att.backward(g, q, k, v, o.clone(), saved=s)[:3]
        assert all(torch.equal(a, b) for a, b in zip(got, w))


@pytest.mark.gpu
def test_refusals():
    cfg = C(2, 50, 80, 2, 64)
    q, k, v, g = _inputs(cfg, 3)
    att = abft.CrossAttention(cfg)
    with pytest.raises(abft.AbftError):         # before any forward
        att.backward(g, q, k, v, torch.zeros_like(q))
    with pytest.raises(abft.AbftError):
        att.backward(g, q, k, v, torch.zeros_like(q), saved=att.new_saved())
    o = att.forward(q, k, v)
    att.backward(g, q, k, v, o)
    att.backward(g, q, k, v, o)                 # twice is fine
    with pytest.raises(abft.AbftError):         # a forward that failed leaves nothing
        att.forward(q, k, v, O=q)
    with pytest.raises(abft.AbftError):
        att.backward(g, q, k, v, o)
    for other in (C(2, 51, 80, 2, 64), C(2, 50, 80, 2, 128), C(2, 50, 80, 2, 64, dtype="f32")):
        with pytest.raises(abft.AbftError):
            att.forward(q, k, v, saved=abft.CrossAttention(other).new_saved())
    # without a record of its own
    infer = abft.CrossAttention(cfg, training=False)
    o = infer.forward(q, k, v)
    assert infer.lse is None and infer.rest is None
    with pytest.raises(abft.AbftError):
        infer.backward(g, q, k, v, o)
    saved = infer.new_saved()
    o = infer.forward(q, k, v, saved=saved)
    grads = infer.backward(g, q, k, v, o, saved=saved)
    o = att.forward(q, k, v)
    assert all(a is None or torch.equal(a, b)
               for a, b in zip(grads, att.backward(g, q, k, v, o)))
