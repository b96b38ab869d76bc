"""Refusals of the packed sequences' calls, on the host before anything is launched (no GPU needed), and the
rotary's frequencies against the oracle."""

import ctypes
import math

import numpy as np
import pytest

from oracle import packed as oracle_packed

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")

R = ctypes.byref
INVAL, SHAPE, DTYPE, CAPACITY, ALIGN, WORKSPACE = -1, -2, -3, -5, -6, -9
SCALINGS = ["plain", "linear", "base", "rotations", "index"]


def _cache(**kw):
    args = dict(n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, dtype=kvg.KVG_BF16,
                n_pages=8, k_pool=0x1000, v_pool=0x2000)
    args.update(kw)
    return kvg.kvg_cache(**args)


def _seqs(**kw):
    args = dict(batch=2, max_pages=4, max_ctx_len=32, shared_tokens=0, block_tables=0x3000, ctx_lens=0x4000,
                start_pos=0x5000)
    args.update(kw)
    return kvg.kvg_seqs(**args)


def _packed(**kw):
    args = dict(n_tokens=0, max_len=8, cu_tokens=0x6000, q_stride=0, k_stride=0, v_stride=0)
    args.update(kw)
    return kvg.kvg_packed(**args)


def _append(cache=None, seqs=None, packed=None, rotary=None, norm=None, layer0=0, n_layers=2, q=0x10000, k=0x20000,
            v=0x30000, out=0x40000):
    return kvg.raw_call("kvg_norm_append", R(cache or _cache()), R(seqs or _seqs()), R(packed or _packed()),
                        R(rotary or kvg.rotary()), None if norm is None else R(norm), layer0, n_layers, q, k, v, out, None)


def _attn(cache=None, seqs=None, packed=None, layer0=0, n_layers=2, q=0x10000, scale=0.125, out=0x20000, ws=0x30000,
          ws_bytes=None):
    cache, seqs, packed = cache or _cache(), seqs or _seqs(), packed or _packed()
    if ws_bytes is None:
        ws_bytes = kvg.raw_call("kvg_packed_attn_workspace_bytes", R(cache), R(seqs), R(packed), n_layers)
    return kvg.raw_call("kvg_packed_attn", R(cache), R(seqs), R(packed), layer0, n_layers, q, scale, out, ws, ws_bytes, None)


def _rotate(rotary=None, dtype=kvg.KVG_BF16, head_dim=64, n_tokens=0, n_heads=2, pos=0x1000, x=0x10000, xs=0, y=0x20000, ys=0):
    return kvg.raw_call("kvg_rotate", R(rotary or kvg.rotary()), dtype, head_dim, n_tokens, n_heads, pos, x, xs, y, ys, None)


def test_calls_without_tokens_do_nothing():
    assert _append() == 0 and _attn() == 0 and _rotate() == 0
    assert _append(packed=_packed(n_tokens=5, max_len=0)) == 0
    assert _append(q=None, k=None, v=None, out=None) == 0            # an empty tensor has no address
    assert _rotate(x=None, y=None, pos=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(base=1.0), INVAL), (dict(base=-2.0), INVAL), (dict(base=math.nan), INVAL), (dict(base=math.inf), INVAL),
    (dict(amplitude=0.0), INVAL), (dict(amplitude=math.inf), INVAL), (dict(pairing=2), INVAL), (dict(scaling=5), INVAL),
    (dict(scaling=-1), INVAL), (dict(scaling=1, factor=0.5), INVAL), (dict(scaling=2, factor=math.nan), INVAL),
    (dict(scaling=3, factor=2.0, original_len=0.0, fast=2.0, slow=1.0), INVAL),
    (dict(scaling=3, factor=2.0, original_len=10.0, fast=1.0, slow=1.0), INVAL),
    (dict(scaling=4, factor=2.0, original_len=10.0, fast=1.0, slow=0.0), INVAL),
    (dict(rotary_dim=8), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rotary_dim=80), SHAPE), (dict(rotary_dim=24), SHAPE),
])
def test_rotary_refusals(kw, status):
    rt = kvg.rotary(**kw)
    assert _rotate(rotary=rt) == status
    assert _append(rotary=rt) == status
    theta = (ctypes.c_double * 128)()
    assert kvg.raw_call("kvg_rotary_frequencies", R(rt), 64, theta) == status


def test_reserved_and_null_rotary():
    rt = kvg.rotary()
    rt.reserved = 1
    assert _rotate(rotary=rt) == INVAL
    assert kvg.raw_call("kvg_rotate", None, 1, 64, 0, 2, None, None, 0, None, 0, None) == INVAL
    assert kvg.raw_call("kvg_rotary_frequencies", R(kvg.rotary()), 64, None) == INVAL
    assert kvg.raw_call("kvg_rotary_frequencies", R(kvg.rotary()), 96, (ctypes.c_double * 128)()) == SHAPE


def test_rotate_refusals():
    assert _rotate(dtype=kvg.KVG_FP8_E4M3) == DTYPE and _rotate(dtype=9) == DTYPE
    assert _rotate(head_dim=96) == SHAPE
    assert _rotate(n_tokens=-1) == INVAL and _rotate(n_heads=0) == INVAL
    assert _rotate(xs=64) == INVAL                            # rows overlap
    assert _rotate(xs=2 * 64 + 4) == ALIGN                    # rows leave 16 bytes
    assert _rotate(n_tokens=3, x=None) == INVAL and _rotate(n_tokens=3, pos=None) == INVAL
    assert _rotate(n_tokens=3, x=0x10008) == ALIGN and _rotate(n_tokens=3, y=0x10008) == ALIGN
    assert _rotate(n_tokens=3, x=0x10000, y=0x10000, xs=256) == INVAL      # in place: the same rows
    assert _rotate(n_tokens=1 << 25) == SHAPE                 # beyond the grid


@pytest.mark.parametrize("call", [_append, _attn], ids=["append", "attn"])
def test_batch_refusals(call):
    assert call(cache=_cache(head_dim=96)) == SHAPE
    assert call(cache=_cache(dtype=7)) == DTYPE
    assert call(cache=_cache(k_pool=0)) == INVAL
    assert call(layer0=1) == SHAPE
    assert call(seqs=_seqs(batch=0)) == INVAL
    assert call(seqs=_seqs(block_tables=0)) == INVAL
    assert call(seqs=_seqs(max_ctx_len=65)) == CAPACITY       # 4 pages of 16
    assert call(seqs=_seqs(max_pages=(1 << 27))) == SHAPE     # indices past 31 bits
    assert call(packed=_packed(max_len=65)) == CAPACITY
    assert call(packed=_packed(cu_tokens=0)) == INVAL
    assert call(packed=_packed(n_tokens=-1)) == INVAL and call(packed=_packed(max_len=-1)) == INVAL
    assert call(packed=_packed(q_stride=4 * 64 - 8)) == INVAL
    assert call(packed=_packed(q_stride=4 * 64 + 4)) == ALIGN
    some = _packed(n_tokens=3)
    assert call(packed=some, q=0x10002) == ALIGN
    assert call(packed=some, out=0x10008) == ALIGN
    assert call(packed=some, cache=_cache(v_pool=0x2008)) == ALIGN
    assert call(packed=_packed(n_tokens=1 << 25)) == SHAPE


def test_append_refusals():
    some = _packed(n_tokens=3)
    assert _append(packed=_packed(k_stride=64)) == INVAL and _append(packed=_packed(v_stride=2 * 64 + 2)) == ALIGN
    assert _append(packed=some, k=None) == INVAL and _append(packed=some, v=None) == INVAL
    assert _append(q=None) == INVAL and _append(out=None) == INVAL
    assert _append(packed=_packed(n_tokens=3, q_stride=512), out=0x10000) == INVAL    # in place only when dense
    norm = lambda **kw: kvg.kvg_head_norm(**{**dict(q_weight=0x50000, k_weight=0x60000, eps=1e-6, weight_offset=0.0), **kw})  # noqa: E731
    assert _append(norm=norm()) == 0
    assert _append(norm=norm(eps=-1.0)) == INVAL and _append(norm=norm(eps=math.nan)) == INVAL
    assert _append(norm=norm(weight_offset=math.inf)) == INVAL
    assert _append(packed=some, norm=norm(q_weight=0x50008)) == ALIGN


def test_attn_refusals():
    some = _packed(n_tokens=3)
    assert _attn(scale=0.0) == INVAL and _attn(scale=math.nan) == INVAL and _attn(scale=math.inf) == INVAL
    assert _attn(packed=some, q=None) == INVAL and _attn(packed=some, out=None) == INVAL
    assert _attn(packed=some, q=0x10000, out=0x10000) == INVAL
    assert _attn(ws=None) == WORKSPACE and _attn(ws_bytes=0) == WORKSPACE
    assert _attn(packed=some, ws=0x30008) == ALIGN
    many = (ctypes.c_int32 * 130)(*([8] * 130))
    c = _cache(n_layers=130)
    c.layer_window = ctypes.cast(many, ctypes.POINTER(ctypes.c_int32))
    assert _attn(cache=c, n_layers=130) == SHAPE              # windows on too many layers
    many[3] = -1
    assert _attn(cache=c, n_layers=2) == INVAL


def test_workspace_size_of_bad_arguments_is_zero():
    size = lambda c, s, p, n: kvg.raw_call("kvg_packed_attn_workspace_bytes", R(c), R(s), R(p), n)  # noqa: E731
    assert size(_cache(), _seqs(), _packed(), 2) > 0
    assert size(_cache(head_dim=96), _seqs(), _packed(), 2) == 0
    assert size(_cache(), _seqs(batch=0), _packed(), 2) == 0
    assert size(_cache(), _seqs(), _packed(n_tokens=-1), 2) == 0
    assert size(_cache(), _seqs(), _packed(), 0) == 0 and size(_cache(), _seqs(), _packed(), 3) == 0


@pytest.mark.parametrize("scaling", SCALINGS)
@pytest.mark.parametrize("head_dim,dim", [(64, 0), (128, 16), (128, 64), (256, 256), (256, 240)])
def test_frequencies_match_the_oracle(scaling, head_dim, dim):
    kw = dict(factor=6.0, original_len=3000.0, fast=20.0, slow=1.5)
    for base in (10000.0, 500000.0, 37.5):
        rt = kvg.rotary(base, rotary_dim=dim, scaling=SCALINGS.index(scaling), **kw)
        got = kvg.kvg_rotary_frequencies(rt, head_dim)
        want = oracle_packed.frequencies(dim or head_dim, base, scaling, **kw)
        assert len(got) == (dim or head_dim) // 2
        assert np.allclose(got, want, rtol=1e-13, atol=0), np.abs(np.array(got) / want - 1).max()


def test_binding_refuses_wrong_rows():
    torch = pytest.importorskip("torch")
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kvg._token_stride(x[None], 1, 3, 2, 64, torch.float32)
    with pytest.raises(ValueError):
        kvg._token_stride(x.transpose(0, 1)[None], 1, 2, 3, 64, torch.bfloat16)      # heads not dense
    with pytest.raises(ValueError):
        kvg._token_stride(torch.zeros(2, 4, 2, 64)[:, :3], 2, 3, 2, 64, torch.float32)      # layers too far apart
    wide = torch.zeros(2, 3, 5, 64)
    assert kvg._token_stride(wide[:, :, 1:3], 2, 3, 2, 64, torch.float32) == 5 * 64
    assert kvg._token_stride(wide[:, :1, 1:3].contiguous(), 2, 1, 2, 64, torch.float32) == 2 * 64
    with pytest.raises(kvg.KvgError):
        kvg.kvg_rotate(kvg.rotary(), torch.zeros(3, dtype=torch.int64), x.to(torch.float16), x.to(torch.float16))
