"""Dropout from a counter-based generator: the generator against published
results and whole-number arithmetic, which elements stay, their values to the bit,
refusals."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import block_reference as R
from paper_2410_11720_amd import abft

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2410_11720_amd", "csrc")


# ---- host ------------------------------------------------------------------------------

def test_generator_against_its_published_results():
    """The known answers of Philox4x32-10 (counter, key, result) for all bits clear,
    all bits set, and digits of pi."""
    full = 0xFFFFFFFF
    known = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((full,) * 4, (full,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
              (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for ctr, key, want in known:
        assert tuple(int(x) for x in R.philox(ctr, key)) == want
    # the library's, where its counter can be told: row, offset and key are whole words
    word = lambda k, **kw: (abft.attn_dropout_draw(col=2 * k, **kw)
                            | abft.attn_dropout_draw(col=2 * k + 1, **kw) << 16)
    got = [word(k, seed=0, offset=0, site=0, row=0) for k in range(4)]
    assert tuple(got) == known[0][2]


def test_draws_match_whole_number_arithmetic():
    rng = np.random.default_rng(3)
    for _ in range(20):
        seed, offset = (int(x) for x in rng.integers(0, 2 ** 63, 2))
        seed, offset = seed * 2 + 1, offset * 2          # (of all 64 bits)
        site, row0 = int(rng.integers(0, 65536)), int(rng.integers(0, 40))
        want = R.draws(seed, offset, site, row0 + 1, 65536)[row0]
        for col in [0, 1, 7, 8, 65535, *(int(x) for x in rng.integers(0, 65536, 20))]:
            assert abft.attn_dropout_draw(seed, offset, site, row0, col) == want[col]


def test_draw_refusals():
    for site, col in ((65536, 0), (0, 65536)):
        with pytest.raises(abft.AbftError):
            abft.attn_dropout_draw(1, 2, site, 0, col)


DIVIDE = r"""
#include <cstdio>
#include <initializer_list>
#include "divide.hpp"
using namespace abft;
int main() {
  long bad = 0;
  unsigned long x = 88172645463325252ul;
  auto next = [&] { x ^= x << 13; x ^= x >> 7; x ^= x << 17; return x; };
  auto one = [&](unsigned d, unsigned n) {
    if (n < (1u << 31) && Divisor::of(d).quotient(n) != n / d) ++bad;
  };
  for (unsigned d = 1; d < 3000; ++d)
    for (unsigned long k : {0ul, 1ul, 2ul, 3ul, (1ul << 31) / d, (1ul << 31) / d - 1, 1000ul})
      for (long e : {-1l, 0l, 1l}) {
        const long n = long(k * d) + e;
        if (n >= 0) one(d, unsigned(n));
      }
  for (int i = 0; i < 3000000; ++i) {
    const unsigned d = unsigned(next() >> (33 + next() % 31)) | 1;
    const unsigned n = unsigned(next() >> 33);
    one(d, n);
    one(d + 1, n);
    one(d, n / d * d);
    if (n >= d) one(d, n / d * d - 1);
  }
  for (unsigned p = 0; p < 31; ++p) { one(1u << p, 0x7fffffffu); one((1u << p) - (p > 0), 0x7fffffffu); }
  one(0x7fffffffu, 0x7fffffffu); one(0x7fffffffu, 0x7ffffffeu);
  std::printf("%ld\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_division_by_a_product(tmp_path):
    src, exe = tmp_path / "divide.cpp", tmp_path / "divide"
    src.write_text(DIVIDE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout.strip() == "0"


G = 1 << 30


def _t(ptr, stride=(120, 40)):
    return ctypes.byref(abft.Rows(ptr, *stride))


def _status(x=None, res=None, rng=5 * G, y=None, **kw):
    base = dict(batch=2, tokens=3, cols=40, p=0.1)
    base.update(kw)
    return abft._lib.attn_dropout(abft.DropoutConfig(**base).to_c(), x or _t(G), res, rng,
                                  y or _t(2 * G), None)


def test_refusals_before_any_launch():
    """Pointers are never followed: the calls return first."""
    for kw in (dict(batch=-1), dict(tokens=-1), dict(cols=0), dict(p=-0.1), dict(p=1.01),
               dict(p=math.nan), dict(site=65536)):
        assert _status(**kw) == -1, kw
    assert _status(cols=65537) == -2 and _status(batch=2 ** 16, tokens=2 ** 15, y=_t(2 * G, (0, 40))) == -2
    assert _status(rng=None) == -1 and _status(rng=5 * G + 4) == -1
    assert _status(x=_t(0)) == -1 and _status(y=_t(0)) == -1 and _status(x=_t(G + 1)) == -1
    assert _status(x=_t(G, (-1, 40))) == -1 and _status(y=_t(2 * G, (120, 39))) == -1
    assert _status(y=_t(2 * G, (0, 40))) == -1
    assert _status(y=_t(G + 2)) == -1 and _status(res=_t(2 * G + 80)) == -1   # not in place
    assert _status(y=_t(G, (240, 40))) == -1
    assert _status(rng=2 * G + 16) == -1                                      # the state on y
    assert _status(batch=0) == 0 and _status(tokens=0, x=_t(0), y=_t(0)) == 0


def test_python_refusals_without_a_gpu():
    op = abft.Dropout(abft.DropoutConfig(2, 3, 40), device="cpu")
    x = torch.zeros((2, 3, 40), dtype=torch.bfloat16)
    rng = torch.zeros(2, dtype=torch.int64)
    for args in ((x,), (x, rng.int()), (x, rng[:1]), (x.float(), rng), (x[:, :, :39], rng),
                 (x.transpose(1, 2), rng)):
        with pytest.raises(abft.AbftError):
            op.forward(*args)
    with pytest.raises(abft.AbftError):
        op.forward(x, rng, residual=x.float())
    with pytest.raises(abft.AbftError):
        abft.Dropout(abft.DropoutConfig(2, 3, 40, dtype="f16"), device="cpu")


# ---- GPU -------------------------------------------------------------------------------

def _rng(seed, offset):
    wrap = lambda v: v - 2 ** 64 if v >= 2 ** 63 else v
    return torch.tensor([wrap(seed), wrap(offset)], dtype=torch.int64, device="cuda")


def _rows(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(DT[dtype])


SHAPES = [(1, 1, 1), (1, 1, 7), (3, 5, 8), (2, 7, 9), (4, 33, 100), (2, 600, 768), (1, 3, 65536),
          (1, 9, 4099), (50, 1, 16384), (5, 1000, 3)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("p", [0.0, 1e-6, 0.1, 0.5, 0.999, 1.0])
def test_values_to_the_bit(shape, dtype, p):
    print(f"[case] dropout {shape} {dtype} {p}", flush=True)
    seed, offset, site = 0xFEDCBA9876543210, 2 ** 63 + 5, 65535
    op = abft.Dropout(abft.DropoutConfig(*shape, dtype=dtype, p=p, site=site))
    x, res = _rows(shape, dtype, 1), _rows(shape, dtype, 2)
    rng = _rng(seed, offset)
    kept = R.keep(shape, p, (seed, offset), site)
    want = R.dropped(x, kept, p)
    assert torch.equal(op.forward(x, rng, residual=res), (res.float() + want).to(DT[dtype]))
    assert torch.equal(op.forward(x, rng), want.to(DT[dtype]))
    assert torch.equal(op.backward(x, rng), want.to(DT[dtype]))
    if p < 2.0 ** -17:
        assert torch.equal(op.forward(x), x)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_elements_are_zero_whatever_they_held(dtype):
    shape = (2, 5, 333)
    op = abft.Dropout(abft.DropoutConfig(*shape, dtype=dtype, p=0.5))
    kept = R.keep(shape, 0.5, (1, 2), 0)
    x = _rows(shape, dtype, 3)
    x[~kept] = math.nan
    x[:, :, ::2] = torch.where(kept[:, :, ::2], x[:, :, ::2], math.inf)
    y = op.forward(x, _rng(1, 2))
    assert (y[~kept] == 0).all() and torch.equal(y[kept], (x[kept].float() * 2).to(x.dtype))


@pytest.mark.gpu
def test_strides_in_place_and_alignment():
    shape = (3, 4, 45)
    op = abft.Dropout(abft.DropoutConfig(*shape, p=0.3))
    x, res, rng = _rows(shape, "bf16", 4), _rows(shape, "bf16", 5), _rng(7, 8)
    want = op.forward(x, rng, residual=res)
    big = torch.full((6, 5, 50), 3.0, dtype=torch.bfloat16, device="cuda")
    v = big.transpose(0, 1)[1:4, 1:5, 3:48]
    v.copy_(x)
    assert torch.equal(op.forward(v, rng, residual=res), want)
    op.forward(v, rng, residual=res, y=v)
    assert torch.equal(v, want)
    v.fill_(3.0)
    assert (big == 3.0).all()
    y = res.clone()
    assert torch.equal(op.forward(x, rng, residual=y, y=y), want)
    rep = res[:1].expand(shape)
    assert torch.equal(op.forward(x, rng, residual=rep), op.forward(x, rng, residual=rep.contiguous()))


@pytest.mark.gpu
def test_python_refusals():
    op = abft.Dropout(abft.DropoutConfig(2, 3, 40))
    x, rng = _rows((2, 3, 40), "bf16", 7), _rng(1, 2)
    wide = torch.zeros((2, 3, 80), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: op.forward(x), lambda: op.forward(x, rng.int()), lambda: op.forward(x, rng[:1]),
                 lambda: op.forward(x, rng.cpu()), lambda: op.forward(x.float(), rng),
                 lambda: op.forward(x.cpu(), rng), lambda: op.forward(x[:, :, :39], rng),
                 lambda: op.forward(x, rng, residual=x.float()), lambda: op.forward(wide[:, :, ::2], rng),
                 lambda: op.forward(x, rng, y=x.float()), lambda: op.backward(x),
                 lambda: op.forward(wide[:, :, :40], rng, y=wide[:, :, 8:48]),
                 lambda: op.forward(x, rng, y=x[:1].expand(2, 3, 40))):
        with pytest.raises(abft.AbftError):
            call()


@pytest.mark.gpu
def test_what_tells_draws_apart():
    """Other seeds, offsets (high words too), sites and rows draw other masks, whose
    agreement is that of independent ones; a share of t / 65536 is dropped. Bounds of
    six standard deviations of 10^6 draws."""
    shape, p, n = (4, 500, 512), 0.25, 1024000
    x = torch.ones(shape, dtype=torch.bfloat16, device="cuda")

    def mask(seed, offset, site):
        op = abft.Dropout(abft.DropoutConfig(*shape, p=p, site=site))
        return op.forward(x, _rng(seed, offset)) != 0
    first = mask(5, 6, 7)
    assert abs(first.float().mean().item() - 0.75) <= 6 * math.sqrt(p * (1 - p) / n)
    assert torch.equal(first, mask(5, 6, 7))
    same = p * p + (1 - p) * (1 - p)
    for other in (mask(6, 6, 7), mask(5 + 2 ** 32, 6, 7), mask(5, 7, 7), mask(5, 6 + 2 ** 32, 7),
                  mask(5, 6, 8), first.roll(1, dims=1), first.roll(1, dims=2), first.roll(8, dims=2),
                  first.roll(1, dims=0)):
        share = (first == other).float().mean().item()
        assert abs(share - same) <= 6 * math.sqrt(same * (1 - same) / n)


@pytest.mark.gpu
def test_captured_calls_draw_anew():
    shape = (2, 100, 768)
    op = abft.Dropout(abft.DropoutConfig(*shape, p=0.1))
    x, rng = _rows(shape, "bf16", 6), _rng(9, 10)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.forward(x, rng, y=y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(x, rng, y=y)
        op.backward(x, rng, dx=dx)
    seen = []
    for _ in range(3):
        rng[1] += 1
        want = op.forward(x, rng)
        y.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, want)
        assert not any(torch.equal(want, s) for s in seen)
        seen.append(want)


@pytest.mark.gpu
def test_more_than_2_to_32_bytes():
    """2.3 G elements in place: the last rows are right."""
    shape = (3, 12000, 65536)
    op = abft.Dropout(abft.DropoutConfig(*shape, p=0.5, site=1))
    x = torch.ones(shape, dtype=torch.bfloat16, device="cuda")
    op.forward(x, _rng(3, 4), y=x)
    cols = [0, 1, 9, 40000, *range(65500, 65536)]
    for row in (0, 17000, 35999):
        u = np.array([abft.attn_dropout_draw(3, 4, 1, row, c) for c in cols])
        got = x.view(-1, 65536)[row, cols].float().cpu().numpy()
        assert (got == 2.0 * (u >= 32768)).all()
