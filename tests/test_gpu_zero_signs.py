"""Packed attention's zeros: their sign is the same however a row is called."""

import numpy as np
import pytest
import torch

from tests.packed_helpers import TORCH
from tests.test_gpu_packed import bits, kvg  # noqa: F401

pytestmark = pytest.mark.gpu

HKV, LAYERS, D = 16, 4, 64


def build(kvg, dtype, where, room):  # noqa: F811
    """Keys of score 0, whose values are small and negative, and keys 100 to 199 above them (log2 units, over layers and KV heads), whose
    values are 0: a row's sum of values leaves fp32 on the negative side.  `blocks`: the former in keys 0 .. 31, the latter in 32 .. 63.
    `segments`: the latter in keys 0 .. 511, the former in 512 .. 1,023.  Returns (cache, sequences); the first row sees these keys and
    no others."""
    seen = 64 if where == "blocks" else 1024
    light, heavy = (slice(0, 32), slice(32, 64)) if where == "blocks" else (slice(512, 1024), slice(0, 512))
    pages = seen // 16 + 3
    max_pages = -(-(seen - 1 + room + 40) // 16)
    table = np.zeros((1, max_pages), dtype=np.int32)
    table[0, :pages] = np.random.default_rng(3).permutation(pages)
    gap = (100 + 100 * np.arange(LAYERS * HKV) / (LAYERS * HKV)).reshape(LAYERS, 1, HKV)
    step = gap / 1.4426950408889634 / 100                     # of the keys' first dimension
    slots = torch.from_numpy(table[0, :pages].astype(np.int64)).cuda()
    seqs = kvg.Seqs(torch.from_numpy(table).cuda(), torch.tensor([seen - 1], dtype=torch.int32, device="cuda"),
                    torch.zeros(1, dtype=torch.int64, device="cuda"), seen - 1 + room)
    k, v = (np.zeros((LAYERS, pages * 16, HKV, D), dtype=np.float32) for _ in range(2))
    if dtype == "int8":
        k[:, heavy, :, 0] = 100.0
        v[:, light] = -100.0
        cache = kvg.Int8Cache.allocate(LAYERS, pages, 2 * HKV, HKV, D)
        cache.v_scale.fill_(2.0 ** -60)
        cache.k_scale.copy_(torch.from_numpy(step).expand(LAYERS, pages, HKV))
    else:
        k[:, heavy, :, 0] = step * 100
        v[:, light] = -100.0 * 2.0 ** -60
        cache = kvg.Cache.allocate(LAYERS, pages, 2 * HKV, HKV, D, TORCH[dtype])
    for pool, x in ((cache.k_pool, k), (cache.v_pool, v)):
        pool[:, slots] = torch.from_numpy(x.reshape(LAYERS, pages, 16, HKV, D).transpose(0, 1, 3, 2, 4).copy()).cuda().to(pool.dtype)
    return cache, seqs


@pytest.mark.parametrize("where", ["blocks", "segments"])
@pytest.mark.parametrize("dtype", ["int8", "bf16", "f32"])
def test_zeros_have_one_sign(kvg, dtype, where):  # noqa: F811
    """Single tokens, short chunks and tiles, of as many segments as there are and of more."""
    want = None
    for room in (0, 2600):
        cache, seqs = build(kvg, dtype, where, room)
        for n in (1, 16, 40):
            packed = kvg.Packed(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n)
            q = torch.zeros(LAYERS, n, 2 * HKV, D, device="cuda", dtype=cache.raw_dtype)
            q[..., 0] = 1.0
            out = torch.empty_like(q)
            if dtype == "int8":
                kvg.kvg_int8_attn(cache, seqs, packed, 0, LAYERS, q, 1.0, out, kvg.int8_attn_workspace(cache, seqs, packed, LAYERS))
            else:
                kvg.kvg_packed_attn(cache, seqs, packed, 0, LAYERS, q, 1.0, out, kvg.packed_attn_workspace(cache, seqs, packed, LAYERS))
            assert bool(out.isfinite().all()) and bool((out <= 0).all())
            got = bits(out[:, 0])
            want = got if want is None else want
            wrong = (got != want).any(dim=2).nonzero()
            assert len(wrong) == 0, f"room {room}, {n} rows: (layer, head) {wrong[:8].tolist()} of {len(wrong)}"
