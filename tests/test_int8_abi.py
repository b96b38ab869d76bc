"""Int8 caches: refusals on the host before anything is launched, sizes and headers (no GPU needed), the binding's checks and the
oracle's page."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import int8 as oracle

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")

R = ctypes.byref
INVAL, SHAPE, DTYPE, POSITION, CAPACITY, ALIGN, CORRUPT, WORKSPACE = -1, -2, -3, -4, -5, -6, -7, -9


def _pages(**kw):
    args = dict(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, dtype=kvg.KVG_INT8, n_pages=8, k_pool=0x1000,
                v_pool=0x2000)
    args.update(kw)
    return kvg.kvg_cache(**args)


def _cache(k_scale=0x8000, v_scale=0x9000, **kw):
    return kvg.kvg_int8_cache(_pages(**kw), k_scale, v_scale)


def _seqs(**kw):
    args = dict(batch=2, max_pages=4, max_ctx_len=32, shared_tokens=0, block_tables=0x3000, ctx_lens=0x4000, start_pos=0x5000)
    args.update(kw)
    return kvg.kvg_seqs(**args)


def _packed(**kw):
    args = dict(n_tokens=0, max_len=8, cu_tokens=0x6000, q_stride=0, k_stride=0, v_stride=0)
    args.update(kw)
    return kvg.kvg_packed(**args)


def _append(cache=None, seqs=None, packed=None, rotary=None, axes=None, norm=None, layer0=0, n_layers=2, q=0x10000, k=0x20000,
            v=0x30000, out=0x40000):
    return kvg.raw_call("kvg_int8_append", R(cache or _cache()), R(seqs or _seqs()), R(packed or _packed()), R(rotary or kvg.rotary()),
                        None if axes is None else R(axes), None if norm is None else R(norm), layer0, n_layers, q, k, v, out, None)


def _attn(cache=None, seqs=None, packed=None, layer0=0, n_layers=2, q=0x10000, scale=0.125, out=0x20000, ws=0x30000, ws_bytes=None):
    cache, seqs, packed = cache or _cache(), seqs or _seqs(), packed or _packed()
    if ws_bytes is None:
        ws_bytes = kvg.raw_call("kvg_int8_attn_workspace_bytes", R(cache), R(seqs), R(packed), n_layers)
    return kvg.raw_call("kvg_int8_attn", R(cache), R(seqs), R(packed), layer0, n_layers, q, scale, out, ws, ws_bytes, None)


def test_calls_without_tokens_do_nothing():
    assert _append() == 0 and _attn() == 0
    assert _append(packed=_packed(n_tokens=5, max_len=0)) == 0
    assert _append(q=None, k=None, v=None, out=None) == 0


@pytest.mark.parametrize("call", [_append, _attn], ids=["append", "attn"])
def test_refusals(call):
    for dtype in (kvg.KVG_F32, kvg.KVG_BF16, kvg.KVG_FP8_E4M3, 4):
        assert call(cache=_cache(dtype=dtype)) == DTYPE
    assert call(cache=_cache(k_scale=None)) == INVAL and call(cache=_cache(v_scale=None)) == INVAL
    assert call(cache=_cache(head_dim=96)) == SHAPE and call(cache=_cache(page_size=32)) == SHAPE
    assert call(cache=_cache(n_q_heads=6)) == SHAPE and call(cache=_cache(k_pool=0)) == INVAL
    assert call(layer0=1) == SHAPE and call(seqs=_seqs(batch=0)) == INVAL and call(seqs=_seqs(max_ctx_len=65)) == CAPACITY
    assert call(packed=_packed(max_len=65)) == CAPACITY and call(packed=_packed(n_tokens=-1)) == INVAL
    assert call(packed=_packed(q_stride=4 * 64 - 8)) == INVAL and call(packed=_packed(q_stride=4 * 64 + 4)) == ALIGN
    some = _packed(n_tokens=3)
    assert call(packed=some, q=0x10002) == ALIGN and call(packed=some, out=0x10008) == ALIGN
    assert call(packed=some, cache=_cache(v_pool=0x2008)) == ALIGN


def test_append_refusals():
    some = _packed(n_tokens=3)
    assert _append(packed=_packed(k_stride=64)) == INVAL and _append(packed=_packed(v_stride=2 * 64 + 2)) == ALIGN
    assert _append(packed=some, k=None) == INVAL and _append(q=None) == INVAL and _append(out=None) == INVAL
    axes = kvg.kvg_axes(0x7000, 3, 0, 0, 0, (ctypes.c_int32 * 4)(8, 12, 12))
    assert _append(axes=axes) == 0
    axes.pairs[0] = 9
    assert _append(axes=axes) == SHAPE
    axes.n_axes = 9
    assert _append(axes=axes) == INVAL
    assert _append(rotary=kvg.rotary(base=0.5)) == INVAL
    assert _append(norm=kvg.kvg_head_norm(0x50000, 0x60000, -1.0, 0.0)) == INVAL
    assert _append(packed=some, norm=kvg.kvg_head_norm(0x50008, 0x60000, 1e-6, 0.0)) == ALIGN


def test_attn_refusals():
    some = _packed(n_tokens=3)
    assert _attn(scale=0.0) == INVAL and _attn(scale=float("nan")) == INVAL
    assert _attn(packed=some, q=None) == INVAL and _attn(packed=some, q=0x10000, out=0x10000) == INVAL
    assert _attn(ws=None) == WORKSPACE and _attn(ws_bytes=0) == WORKSPACE and _attn(packed=some, ws=0x30008) == ALIGN
    size = lambda c, n: kvg.raw_call("kvg_int8_attn_workspace_bytes", R(c), R(_seqs()), R(_packed(n_tokens=4)), n)  # noqa: E731
    assert size(_cache(), 2) > 0 and size(_cache(), 3) == 0 and size(_cache(dtype=kvg.KVG_BF16), 2) == 0


def test_other_calls_refuse_int8_pages():
    c, s, p = _pages(), _seqs(), _packed()
    assert kvg.raw_call("kvg_norm_append", R(c), R(s), R(p), R(kvg.rotary()), None, 0, 2, 0x10000, 0x20000, 0x30000, 0x40000, None) == DTYPE
    assert kvg.raw_call("kvg_packed_attn", R(c), R(s), R(p), 0, 2, 0x10000, 0.1, 0x20000, 0x30000, 1 << 30, None) == DTYPE
    assert kvg.raw_call("kvg_append", R(c), R(s), R(kvg.rope()), 0, 2, 1, 0x10000, 0x20000, None) == DTYPE
    assert kvg.raw_call("kvg_decode_workspace_bytes", R(c), R(s), 2) == 0
    assert kvg.raw_call("kvg_deposit", R(c), 0x3000, 4, 0, 16, 0x10000, None) == DTYPE
    assert kvg.raw_call("kvg_payload_bytes", R(c), 16) == 0
    hdr = kvg.kvg_artifact_hdr()
    assert kvg.raw_call("kvg_artifact_header_init", R(c), 16, 0, R(kvg.rope()), R(hdr)) == DTYPE


def _hdr(cache, n=40, own=0):
    hdr = kvg.kvg_artifact_hdr()
    assert kvg.raw_call("kvg_int8_header_init", R(cache), n, own, R(hdr)) == 0
    return hdr


def _graft(cache, hdr, payload=0x10000, table=0x3000, table_len=4, first=0, target=0):
    return kvg.raw_call("kvg_int8_graft", R(cache), R(hdr), payload, table, table_len, first, target, None)


def _deposit(cache, table=0x3000, table_len=4, first=0, n=40, payload=0x10000):
    return kvg.raw_call("kvg_int8_deposit", R(cache), table, table_len, first, n, payload, None)


def test_blocks():
    c = _cache()
    size = lambda n: kvg.raw_call("kvg_int8_payload_bytes", R(c), n)  # noqa: E731
    assert size(40) == 2 * 2 * 3 * 2 * (16 * 64 + 4) and size(0) == 0 and size(2 ** 31 - 1) == 2 * 2 * 2 ** 27 * 2 * (16 * 64 + 4)
    h = _hdr(c, own=7)
    assert (h.dtype, h.own_pos, h.n_tokens, h.rope_pairing, h.payload_bytes) == (kvg.KVG_INT8, 7, 40, kvg.KVG_ROPE_OTHER, size(40))
    assert kvg.raw_call("kvg_artifact_digest_workspace_bytes", R(h)) > 0
    h.payload_bytes -= 4
    assert kvg.raw_call("kvg_artifact_digest_workspace_bytes", R(h)) == 0
    assert _graft(c, h, target=7) == CORRUPT
    h = _hdr(c, own=7)
    assert _graft(c, h, target=8) == POSITION and _graft(c, h, target=7, first=8) == ALIGN
    assert _graft(c, h, target=7, table_len=2) == CAPACITY and _graft(c, h, target=7, first=32) == CAPACITY
    assert _graft(c, h, payload=0x10008, target=7) == ALIGN and _graft(c, h, payload=None, target=7) == INVAL
    assert _graft(_cache(k_scale=None), h, target=7) == INVAL and _graft(_cache(dtype=kvg.KVG_FP8_E4M3), h, target=7) == DTYPE
    assert _graft(_cache(head_dim=128), h, target=7) == SHAPE
    h.dtype = kvg.KVG_FP8_E4M3
    assert _graft(c, h, target=7) == DTYPE
    h = _hdr(c)
    h.magic = 1
    assert _graft(c, h) == CORRUPT
    assert _deposit(c, n=0) == INVAL and _deposit(c, first=-16) == INVAL and _deposit(c, first=8) == ALIGN
    assert _deposit(c, table_len=2) == CAPACITY and _deposit(c, payload=0x10004) == ALIGN and _deposit(c, table=None) == INVAL
    assert kvg.raw_call("kvg_int8_header_init", R(c), 0, 0, R(h)) == INVAL
    assert kvg.raw_call("kvg_int8_header_init", R(c), 5, 0, None) == INVAL
    # an int8 block into another cache
    fp8 = _pages(dtype=kvg.KVG_FP8_E4M3)
    assert kvg.raw_call("kvg_graft", R(fp8), R(_hdr(c)), 0x10000, 0x3000, 4, 0, 0, 0, None) == DTYPE


def test_binding_checks():
    pool = torch.zeros(1, 2, 2, 16, 64, dtype=torch.int8)
    scale = torch.zeros(1, 2, 2)
    ok = kvg.Int8Cache(pool, pool.clone(), scale, scale.clone(), 4, (0,))
    assert ok.struct().pages.dtype == kvg.KVG_INT8 and ok.raw_dtype is torch.bfloat16
    windowed = kvg.Int8Cache(pool, pool.clone(), scale, scale.clone(), 4, (9,)).struct()
    assert windowed.pages.layer_window[0] == 9
    for bad in (dict(k_pool=pool.float()), dict(v_pool=pool[:, :1].clone()), dict(k_scale=scale.double()), dict(v_scale=scale[0]),
                dict(k_scale=scale.expand(1, 2, 2).transpose(1, 2)[:, :, :1]), dict(windows=(9, 9))):
        with pytest.raises(ValueError):
            kvg.Int8Cache(**{**dict(k_pool=pool, v_pool=pool.clone(), k_scale=scale, v_scale=scale.clone(), n_q_heads=4), **bad}).struct()
    with pytest.raises(ValueError):
        kvg.kvg_int8_deposit(ok, torch.zeros(2, dtype=torch.int32), 0, 16, torch.zeros(10, dtype=torch.uint8))
    with pytest.raises(ValueError):
        kvg.kvg_int8_deposit(ok, torch.zeros(2, dtype=torch.int64), 0, 16, torch.zeros(9000, dtype=torch.uint8))


def test_oracle_page():
    n, m, s = oracle.append_page(np.array([[100.0, -50.0]]), 0.5, np.array([[127.0, 1.0]]))
    assert s == 1.0 and n.tolist() == [[50.0, -25.0]] and m.tolist() == [[127.0, 1.0]]
    n, m, s = oracle.append_page(np.array([[100.0, -50.0]]), 0.5, np.array([[1.0, 0.25]]))
    assert s == 0.5 and n.tolist() == [[100.0, -50.0]] and m.tolist() == [[2.0, 0.0]]           # ties to even
    n, m, s = oracle.append_page(np.zeros((0, 2)), 9.0, np.zeros((1, 2)))
    assert s == 0.0 and m.tolist() == [[0.0, 0.0]]
    # one key: its value, within the rounding
    q = np.ones((1, 2, 4))
    want, tol = oracle.attend(q, np.array([0]), np.ones((1, 1, 4)), np.ones((1, 1)), np.full((1, 1, 4), 8.0), np.full((1, 1), 0.25), 0.5)
    assert np.allclose(want, 2.0) and np.all(tol < 2 * (2.0 ** -8 + 2.0 ** -10))


def test_oracle_attention():
    """The oracle's attention over integers and scales is the bf16 caches' over the values they stand for."""
    from oracle.packed import attend_bounds
    rng = np.random.default_rng(4)
    kn, vn = (rng.integers(-127, 128, (50, 2, 8)).astype(np.float64) for _ in range(2))
    ks, vs = (np.repeat(rng.random((4, 2)), 16, axis=0)[:50] for _ in range(2))
    q, index = rng.normal(size=(3, 4, 8)), np.array([0, 17, 49])
    for window in (0, 20):
        want = attend_bounds(q, index, kn * ks[..., None], vn * vs[..., None], 0.01, window)[0]
        assert np.allclose(oracle.attend(q, index, kn, ks, vn, vs, 0.01, window)[0], want, rtol=0, atol=1e-12 * np.abs(want).max())
