"""Packed sequences on the GPU at the edges of what their calls allow: blocks of scaled rotaries relocated, values that are not
finite, and single-segment batches of few rows."""

import math

import numpy as np
import pytest
import torch

from oracle import packed as oracle
from tests.packed_helpers import U, Batch, host
from tests.test_gpu_packed import append, bits, make_rotary, pair_size

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    from paper_2607_14431_amd import kvg as k
    return k


# ---------------------------------------------------------------------------- relocated blocks

@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("scaling,dim", [("plain", 0), ("base", 0), ("base", 64), ("linear", 0), ("rotations", 0), ("base", 32)])
def test_blocks_of_scaled_rotaries_relocate_rightly_or_not_at_all(kvg, pairing, scaling, dim):
    """A block's keys turned by d: those of the rotary at the new positions, or a refusal; at its own position its bytes."""
    n, d, D, amplitude = 45, 4099, 64, 1.2
    b = Batch([n], [0], (4, 2, D), "f32", seed=21, poison=3.0)
    rt, theta = make_rotary(kvg, D, pairing, dim, scaling, amplitude=amplitude)
    k, v = b.rows(2), b.rows(2)
    append(b, rt, None, None, k, v, None)
    start = int(b.start[0])
    hdr = kvg.kvg_artifact_header_init_rotary(b.cache, n, start, rt)
    payload = torch.empty(hdr.payload_bytes, dtype=torch.uint8, device="cuda")
    kvg.kvg_deposit(b.cache, b.seqs.block_tables[0], 0, n, payload)
    there = Batch([n], [0], (4, 2, D), "f32", seed=22, poison=3.0)
    kvg.kvg_graft(there.cache, hdr, payload, there.seqs.block_tables[0], 0, start)
    for got, want in zip(there.keys_values(0, 0), b.keys_values(0, 0)):
        assert np.array_equal(got, want)
    move = lambda: kvg.kvg_graft(there.cache, hdr, payload, there.seqs.block_tables[0], 0, start + d,  # noqa: E731
                                 kvg.KVG_GRAFT_ALLOW_RELOCATE)
    if scaling in ("linear", "rotations") or dim not in (0, D):
        with pytest.raises(kvg.KvgError, match="position"):
            move()
        return
    move()
    want = oracle.rotate(host(k[0]), start + d + np.arange(n), theta, pairing, amplitude)
    size = amplitude * pair_size(host(k[0]), D, pairing)
    # a rotation in fp32 is off by 4 u of the pair's size (cos and sin sqrt 2, a product and the sum 2, rounded up) and its
    # stored value by u more; the second rotation takes in the first one's error from both components (sqrt 2 of it)
    assert np.all(np.abs(there.keys_values(0, 0)[0] - want) <= 5 * U * (1 + math.sqrt(2)) * 1.01 * size)
    assert np.array_equal(there.keys_values(0, 0)[1], b.keys_values(0, 0)[1])
