"""Attention over keys of another length refuses outputs that share memory with
another argument, and tells views that only interleave apart from them."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2410_11720_amd import abft

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2410_11720_amd", "csrc")
C = abft.CrossConfig

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "overlap.hpp"
using namespace abft;

static uint64_t state = 88172645463325252ull;
static int pick(int n) {
  state ^= state << 13; state ^= state >> 7; state ^= state << 17;
  return int(state % uint64_t(n));
}

static void bytes(const Area& a, std::vector<char>& mem) {
  if (a.end == a.at) return;
  for (int64_t x = 0; x <= a.last[0]; ++x)
    for (int64_t y = 0; y <= a.last[1]; ++y)
      for (int64_t z = 0; z <= a.last[2]; ++z)
        for (int64_t e = 0; e < a.row; ++e)
          mem[a.at + x * a.stride[0] + y * a.stride[1] + z * a.stride[2] + e] = 1;
}

int main() {
  long bad = 0, met = 0, apart = 0;
  for (int n = 0; n < 200000; ++n) {
    Area a[2];
    // one packed layout, or one of its own each; dimensions in any order
    const int row = 1 + pick(4), heads = 1 + pick(3), tokens = 1 + pick(3);
    int64_t st[3] = {row * (1 + pick(4)), 0, 0};
    st[1] = st[0] * heads + pick(3);
    st[2] = st[1] * tokens * (1 + pick(2));
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && pick(3) == 0)
        for (auto& s : st) s = pick(30);
      a[k] = Area::flat(reinterpret_cast<void*>(uintptr_t(64 + pick(60))), size_t(1 + pick(row + 1)));
      a[k].dim(0, st[2], pick(3));
      a[k].dim(1, st[1], 1 + pick(tokens + 1));
      a[k].dim(2, st[0], 1 + pick(heads + 1));
    }
    std::vector<char> m0(2048), m1(2048);
    bytes(a[0], m0);
    bytes(a[1], m1);
    bool want = false;
    for (size_t x = 0; x < m0.size(); ++x) want = want || (m0[x] && m1[x]);
    if (overlap(a[0], a[1]) != want || overlap(a[1], a[0]) != want) ++bad;
    ++(want ? met : apart);
  }
  // three thirds of a packed tensor with 2^40 rows, in few steps
  Area big[3];
  for (int k = 0; k < 3; ++k) {
    big[k] = Area::flat(reinterpret_cast<void*>(uintptr_t(4096 + 1280 * k)), 128);
    big[k].dim(0, int64_t(3840) << 24, 1 << 12);
    big[k].dim(1, 3840, 1 << 24);
    big[k].dim(2, 128, 10);
  }
  if (overlap(big[0], big[1]) || overlap(big[1], big[2]) || overlap(big[0], big[2])) ++bad;
  big[1].last[2] = 10;  // a head into the last third
  if (!overlap(big[1], big[2]) || overlap(big[0], big[1])) ++bad;
  std::printf("%ld wrong, %ld met, %ld apart\n", bad, met, apart);
  return bad != 0 || met < 1000 || apart < 1000;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_overlap_against_every_byte(tmp_path):
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout


# ---- refusals: addresses that are never followed -----------------------------------

QS, KS = (2, 3, 5, 64), (2, 5, 5, 64)       # 3840 and 6400 bytes in bf16
WS = 1 << 40


def _t(at, shape, stride=None):
    if stride is None:
        stride = (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])
    return ctypes.byref(abft.CrossTensor(at, *stride))


def _forward(O=0x50000, lse=0x60000, rest=0x70000, bias=0x80000, ws=WS):
    c = C(2, 3, 5, 5, 64, buckets=32).to_c()
    return abft._lib.attn_cross_forward(
        c, _t(0x10000, QS), _t(0x20000, KS), _t(0x30000, KS), bias, 0x90000, 0xa0000, _t(O, QS),
        lse, rest, ws, 1 << 30, None)


def _backward(dQ=0x1000000, dK=0x2000000, dV=0x3000000, dbias=0x4000000, ws=WS, dq_stride=None):
    c = C(2, 3, 5, 5, 64, buckets=32).to_c()
    return abft._lib.attn_cross_backward(
        c, _t(0x40000, QS), _t(0x10000, QS), _t(0x20000, KS), _t(0x30000, KS), _t(0x50000, QS),
        0x60000, 0x70000, 0x80000, 0x90000, 0xa0000, _t(dQ, QS, dq_stride), _t(dK, KS), _t(dV, KS),
        dbias, ws, 1 << 30, None)


def test_forward_refuses_what_shares_memory():
    # O on Q, on the last row of K, on V's first; lse, rest, workspace on others
    for at in (0x10000, 0x20000 + 6400 - 16, 0x30000 - 3840 + 16, 0x80010, 0x90000 - 3824):
        assert _forward(O=at) == -1, hex(at)
    assert _forward(lse=0x50000) == -1 and _forward(lse=0xa0000) == -1
    assert _forward(rest=0x60000) == -1 and _forward(rest=0x10000) == -1
    c = C(1, 1, 8192, 1, 64).to_c()          # (keys split over workgroups: partial results)
    q, k = (1, 1, 1, 64), (1, 8192, 1, 64)
    for ws in (0x10000, 0x200000, 0x50000):
        assert abft._lib.attn_cross_forward(c, _t(0x10000, q), _t(0x200000, k), _t(0x400000, k),
                                            None, None, None, _t(0x50000, q), None, None, ws,
                                            1 << 30, None) == -1


def test_backward_refuses_what_shares_memory():
    # on each input, on another output, on the workspace
    for at in (0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000, 0x80000, 0x90000,
               0xa0000, 0x2000000 + 6384, 0x4000000, WS):
        assert _backward(dQ=at) == -1, hex(at)
    assert _backward(dK=0x3000000) == -1 and _backward(dV=0x2000000 + 6384) == -1
    assert _backward(dbias=0x1000000) == -1 and _backward(dbias=0x80000) == -1
    assert _backward(ws=0x2000000) == -1 and _backward(ws=0x60000) == -1
    # rows of two packed outputs that do meet: dK starts inside dQ's second third
    assert _backward(dQ=0x2000000 - 1920 + 16, dq_stride=(3 * 960, 960, 64)) == -1


def test_strides_that_no_memory_has():
    c = C(2, 3, 5, 5, 64).to_c()
    for st in ((2 ** 62, 320, 64), (2 ** 56, 320, 64), (960, 320, 2 ** 60)):
        assert abft._lib.attn_cross_forward(
            c, _t(0x10000, QS, st), _t(0x20000, KS), _t(0x30000, KS), None, None, None,
            _t(0x50000, QS), None, None, WS, 1 << 30, None) == -1


# ---- GPU ------------------------------------------------------------------------------

@pytest.mark.gpu
def test_packed_views_are_not_refused():
    """Inputs and outputs, forward and backward, in one buffer, rows interleaved."""
    B, S, nh, d = 2, 70, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    box = torch.randn((B, S, 8, nh, d), generator=gen, device="cuda").bfloat16()
    q, k, v, g, o, dq, dk, dv = box.unbind(2)
    att = abft.CrossAttention(C(B, S, S, nh, d, causal=True))
    att.forward(q, k, v, O=o)
    att.backward(g, q, k, v, o, dQ=dq, dK=dk, dV=dv)
    apart = [t.clone() for t in (q, k, v, g)]
    o2 = att.forward(*apart[:3])
    grads = att.backward(apart[3], *apart[:3], o2)
    for a, b in zip((o, dq, dk, dv), (o2, *grads)):
        assert torch.equal(a, b)
    # key heads beside query heads in one buffer, of other extents and strides
    heads = torch.randn((B, 12, S, d), generator=gen, device="cuda").bfloat16()
    q, o = (heads[:, i:i + 4].transpose(1, 2) for i in (0, 8))
    k, v = (heads[:, i:i + 2].transpose(1, 2) for i in (4, 6))
    att = abft.CrossAttention(C(B, S, S, 4, d, kv_heads=2))
    want = att.forward(q.clone(), k.clone(), v.clone())
    assert torch.equal(att.forward(q, k, v, O=o), want)


@pytest.mark.gpu
def test_shared_outputs_are_refused():
    cfg = C(2, 70, 70, 4, 64)
    q, k, v, g = (torch.randn((2, 70, 4, 64), device="cuda").bfloat16() for _ in range(4))
    att = abft.CrossAttention(cfg)
    o = att.forward(q, k, v)
    buf = torch.empty_like(k)
    with pytest.raises(abft.AbftError):
        att.forward(q, k, v, O=q)
    for kw in (dict(dK=buf, dV=buf), dict(dQ=g), dict(dQ=q), dict(dV=v), dict(dK=o)):
        with pytest.raises(abft.AbftError):
            att.backward(g, q, k, v, o, **kw)
