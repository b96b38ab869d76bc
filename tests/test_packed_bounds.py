"""Packed sequences at the edges of what their arguments allow, on the host before anything is launched (no GPU needed)."""

import ctypes

import pytest

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")

R = ctypes.byref
ALIGN, WORKSPACE = -6, -9


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


@pytest.mark.parametrize("zeros", [False, True], ids=["no windows", "windows of 0"])
@pytest.mark.parametrize("layers", [128, 129, 130, 256, 700])
@pytest.mark.parametrize("heads,tokens,ctx", [(1, 64, 32000), (2, 300, 8000), (8, 40, 3000)])
def test_plan_of_many_layers_is_the_size_querys(layers, heads, tokens, ctx, zeros):
    """More layers than a launch carries windows of, none of them windowed: the call plans as the size query did.  Its
    workspace of exactly that size is refused for its address alone, one byte less for its size."""
    c = _cache(n_layers=layers, n_q_heads=heads, n_kv_heads=heads, n_pages=4096)
    if zeros:
        none = (ctypes.c_int32 * layers)()
        c.layer_window = ctypes.cast(none, ctypes.POINTER(ctypes.c_int32))
    s, p = _seqs(batch=1, max_pages=4000, max_ctx_len=ctx), _packed(n_tokens=tokens, max_len=tokens)
    size = kvg.raw_call("kvg_packed_attn_workspace_bytes", R(c), R(s), R(p), layers)
    assert size > 0
    call = lambda n: kvg.raw_call("kvg_packed_attn", R(c), R(s), R(p), 0, layers, 0x10000, 0.125, 0x20000, 0x30008, n, None)  # noqa: E731
    for _ in range(3):
        assert call(size) == ALIGN
        assert call(size - 1) == WORKSPACE


def test_rotate_refuses_rows_that_overlap():
    """A row broadcast over tokens has stride 0, which the library takes for dense rows: refused, as rows that overlap."""
    torch = pytest.importorskip("torch")
    pos = torch.zeros(5, dtype=torch.int64)
    dense = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    broadcast = torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(5, 2, 64)
    sliding = torch.zeros(6 * 64, dtype=torch.bfloat16).as_strided((5, 2, 64), (64, 64, 1))
    one_head = torch.zeros(1, 1, 64).expand(5, 1, 64)
    for x, y in ((broadcast, dense), (dense, broadcast), (broadcast, broadcast), (sliding, dense), (dense, sliding),
                 (one_head, torch.zeros(5, 1, 64))):
        with pytest.raises(ValueError, match="overlap"):
            kvg.kvg_rotate(kvg.rotary(), pos, x, y)
