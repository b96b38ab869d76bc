"""Positions with several axes: refusals on the host before anything is launched (no GPU needed), the binding's checks, and
the oracle's definition."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import packed as oracle

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")

R = ctypes.byref
INVAL, SHAPE = -1, -2


def _axes(pairs=(8, 12, 12), **kw):
    args = dict(positions=0x1000, n_axes=len(pairs), order=0, own_frequencies=0, reserved=0)
    args.update(kw)
    return kvg.kvg_axes(pairs=(ctypes.c_int32 * 4)(*pairs), **args)


def _rotate(axes, rotary=None, n_tokens=0, head_dim=64):
    return kvg.raw_call("kvg_rotate_axes", R(rotary or kvg.rotary()), None if axes is None else R(axes), 1, head_dim, n_tokens, 2,
                        0x10000, 0, 0x20000, 0, None)


def _append(axes, rotary=None, n_tokens=0):
    cache = kvg.kvg_cache(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, dtype=kvg.KVG_BF16, n_pages=8,
                          k_pool=0x1000, v_pool=0x2000)
    seqs = kvg.kvg_seqs(batch=2, max_pages=4, max_ctx_len=32, shared_tokens=0, block_tables=0x3000, ctx_lens=0x4000, start_pos=0x5000)
    packed = kvg.kvg_packed(n_tokens=n_tokens, max_len=8, cu_tokens=0x6000, q_stride=0, k_stride=0, v_stride=0)
    return kvg.raw_call("kvg_norm_append_axes", R(cache), R(seqs), R(packed), R(rotary or kvg.rotary()),
                        None if axes is None else R(axes), None, 0, 2, 0x10000, 0x20000, 0x30000, 0x40000, None)


@pytest.mark.parametrize("call", [_rotate, _append], ids=["rotate", "append"])
def test_refusals(call):
    assert call(_axes()) == 0 and call(_axes((32,))) == 0 and call(_axes((1, 1, 1, 29), order=1)) == 0
    assert call(_axes(), rotary=kvg.rotary(rotary_dim=48)) == SHAPE and call(_axes((8, 8, 8)), rotary=kvg.rotary(rotary_dim=48)) == 0
    assert call(None) == INVAL
    assert call(_axes(n_axes=0)) == INVAL and call(_axes(n_axes=5)) == INVAL and call(_axes(reserved=1)) == INVAL
    assert call(_axes(order=2)) == INVAL and call(_axes(order=-1)) == INVAL
    assert call(_axes(own_frequencies=1)) == 0
    assert call(_axes(own_frequencies=2)) == INVAL and call(_axes(own_frequencies=1, order=1)) == INVAL
    assert call(_axes((0, 16, 16))) == SHAPE and call(_axes((-8, 20, 20))) == SHAPE
    assert call(_axes((8, 12, 11))) == SHAPE and call(_axes((2 ** 31 - 1, 2 ** 31 - 1, 34))) == SHAPE
    based = kvg.rotary(scaling=kvg.KVG_ROTARY_BASE, factor=2.0)
    assert call(_axes((1, 15, 16)), rotary=based) == 0
    assert call(_axes((1, 15, 16), own_frequencies=1), rotary=based) == SHAPE
    assert call(_axes((2, 14, 16), own_frequencies=1), rotary=based) == 0
    assert call(_axes(positions=None)) == 0 and call(_axes(positions=None), n_tokens=3) == INVAL


def test_binding_checks():
    pos = torch.zeros(3, 5, dtype=torch.int64)
    assert kvg.Axes(pos, (8, 12, 12)).struct(5).n_axes == 3
    for bad, pairs in ((pos[:, :4], (8, 12, 12)), (pos.int(), (8, 12, 12)), (pos, (16, 16)), (pos.t().contiguous().t(), (8, 12, 12)),
                       (torch.zeros(5, 5, dtype=torch.int64), (8, 6, 6, 6, 6)), (pos[:0], ())):
        with pytest.raises(ValueError):
            kvg.Axes(bad, pairs).struct(5)
    x = torch.zeros(5, 2, 64)
    with pytest.raises(ValueError):
        kvg.kvg_rotate_axes(kvg.rotary(), kvg.Axes(pos, (8, 12, 12)), x[:1].expand(5, 2, 64), x)      # rows overlap
    with pytest.raises(kvg.KvgError):
        kvg.kvg_rotate_axes(kvg.rotary(), kvg.Axes(pos, (8, 12, 12)), x.half(), x.half())


def test_oracle_axes():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(7, 2, 64))
    assert oracle.axis_of_pairs((2, 3), "sections").tolist() == [0, 0, 1, 1, 1]
    assert oracle.axis_of_pairs((4, 2, 1), "turns").tolist() == [0, 1, 2, 0, 1, 0, 0]
    theta = oracle.frequencies(64, 10000.0)
    same = np.tile(rng.integers(0, 999, 7), (3, 1))
    for order in ("sections", "turns"):                       # one position on every axis: a plain rotary
        axis = oracle.axis_of_pairs((12, 10, 10), order)
        assert np.allclose(oracle.rotate_axes(x, same, theta, axis, "half"), oracle.rotate(x, same[0], theta, "half"), atol=1e-12)
    # each axis' own frequencies, interleaved: a rotary of its own on its part of the head
    pos = rng.integers(0, 999, (2, 7))
    got = oracle.rotate_axes(x, pos, oracle.axes_frequencies((20, 12), 10000.0, True), oracle.axis_of_pairs((20, 12), "sections"), "interleaved")
    for lo, hi, p in ((0, 40, pos[0]), (40, 64, pos[1])):
        part = oracle.rotate(x[..., lo:hi], p, oracle.frequencies(hi - lo, 10000.0), "interleaved")
        assert np.allclose(got[..., lo:hi], part, atol=1e-12)
