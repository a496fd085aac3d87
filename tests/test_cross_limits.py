"""Attention over keys of another length: calls whose grids are out of HIP's range
(2^32 threads) are refused before anything is launched. Addresses that are never
followed."""
import ctypes

import pytest

from paper_2410_11720_amd import abft

C = abft.CrossConfig
G = 1 << 40


def _t(k, shape):
    st = (shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])
    return ctypes.byref(abft.CrossTensor(k * G, *st))


def _both(cfg):
    c = cfg.to_c()
    qs = (cfg.batch, cfg.q_len, cfg.heads, cfg.head_dim)
    ks = (cfg.batch, cfg.k_len, cfg.kv_heads or cfg.heads, cfg.head_dim)
    bias = 15 * G if cfg.buckets else None
    forward = abft._lib.attn_cross_forward(c, _t(1, qs), _t(2, ks), _t(3, ks), bias, None, None,
                                           _t(4, qs), 5 * G, None, 16 * G, 1 << 40, None)
    backward = abft._lib.attn_cross_backward(c, _t(6, qs), _t(1, qs), _t(2, ks), _t(3, ks),
                                             _t(4, qs), 5 * G, None, bias, None, None, _t(7, qs),
                                             _t(8, ks), _t(9, ks), 14 * G if bias else None, 16 * G,
                                             1 << 40, None)
    return forward, backward


@pytest.mark.parametrize("cfg,want", [
    (C(1 << 20, 1, 1, 16, 64), (-2, -2)),                 # 2^24 workgroups of 256
    (C(1 << 20, 100, 40, 16, 128), (-2, -2)),
    (C(1 << 20, 1, 1, 16, 64, dtype="f32", buckets=32), (-2, -2)),
    (C(1, 1, 1, 1 << 24, 64, buckets=2, max_distance=2, bidirectional=False), (-2, -2)),
], ids=str)
def test_grids_out_of_range(cfg, want):
    assert _both(cfg) == want


def test_key_pass_alone_out_of_range():
    """2^23 workgroups of eight waves; the forward's grid is in range."""
    cfg = C(1 << 19, 1, 200, 16, 128)
    c = cfg.to_c()
    qs, ks = (cfg.batch, 1, 16, 128), (cfg.batch, 200, 16, 128)
    assert abft._lib.attn_cross_backward(c, _t(6, qs), _t(1, qs), _t(2, ks), _t(3, ks), _t(4, qs),
                                         5 * G, None, None, None, None, _t(7, qs), _t(8, ks),
                                         _t(9, ks), None, 16 * G, 1 << 40, None) == -2
