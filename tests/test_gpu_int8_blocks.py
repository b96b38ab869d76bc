"""Blocks of int8 caches (deposit, digest, file, graft), captured calls, other streams, and a run of the serving step's calls
together."""

import math

import numpy as np
import pytest
import torch

from oracle import digest as oracle_digest
from tests.int8_helpers import Int8Batch, check
from tests.packed_helpers import host
from tests.test_gpu_packed import bits, kvg  # noqa: F401

pytestmark = pytest.mark.gpu


def other_cache(kvg, b, fill=99):  # noqa: F811
    """An empty cache of b's geometry, and a table of other pages for sequence 0."""
    c = kvg.Int8Cache.allocate(b.layers, b.cache.n_pages, *b.heads, windows=b.windows)
    for t in c.tensors():
        t.fill_(fill)
    table = torch.from_numpy(np.random.default_rng(77).permutation(b.cache.n_pages)[:b.max_pages].astype(np.int32)).cuda()[None]
    return c, table.contiguous()


@pytest.mark.parametrize("heads,layers,n", [((4, 2, 64), 2, 40), ((2, 1, 128), 1, 1), ((16, 8, 256), 3, 160), ((4, 4, 64), 1, 16)])
def test_deposit_graft(kvg, heads, layers, n):  # noqa: F811
    b = Int8Batch([1], [n + 30], heads, layers, seed=4)
    row = b.seqs.block_tables[0]
    size = kvg.kvg_int8_payload_bytes(b.cache, n)
    payload = torch.full((size + 16,), 55, dtype=torch.uint8, device="cuda")
    kvg.kvg_int8_deposit(b.cache, row, 16, n, payload)
    assert bool((payload[size:] == 55).all())
    pages = -(-n // 16)
    ids = row[1:1 + pages].long()
    Hkv, D = heads[1], heads[2]
    want = torch.stack([b.cache.k_pool[:, ids], b.cache.v_pool[:, ids]], dim=1)       # [L][2][pages][Hkv][16][D]
    if n % 16:
        want[:, :, -1, :, n % 16:] = 0
    split = size - layers * 2 * pages * Hkv * 4
    assert torch.equal(payload[:split].view(torch.int8).view(want.shape), want)
    scales = torch.stack([b.cache.k_scale[:, ids], b.cache.v_scale[:, ids]], dim=1)
    assert torch.equal(payload[split:size].view(torch.float32).view(scales.shape), scales)

    hdr = kvg.kvg_int8_header_init(b.cache, n, 1016)
    c, table = other_cache(kvg, b)
    before = [t.clone() for t in c.tensors()]
    kvg.kvg_int8_graft(c, hdr, payload, table[0], 16, 1016)
    to = table[0, 1:1 + pages].long()
    for pool, was, j in ((c.k_pool, before[0], 0), (c.v_pool, before[1], 1)):
        got = pool[:, to]
        if n % 16:
            assert torch.equal(got[:, -1, :, n % 16:], was[:, to][:, -1, :, n % 16:])      # rows past the block
            got = got.clone()
            got[:, -1, :, n % 16:] = 0
        assert torch.equal(got, want[:, j])
        was[:, to] = pool[:, to]
        assert torch.equal(pool, was)                                                       # no other page
    for s, was, j in ((c.k_scale, before[2], 0), (c.v_scale, before[3], 1)):
        was[:, to] = scales[:, j]
        assert torch.equal(s, was)
    with pytest.raises(kvg.KvgError):
        kvg.kvg_int8_graft(c, hdr, payload, table[0], 16, 1017)


def test_digest_and_file(kvg, tmp_path):  # noqa: F811
    from paper_2607_14431_amd import harness
    b = Int8Batch([1], [70], (4, 2, 64), 2, seed=4)
    hdr = kvg.kvg_int8_header_init(b.cache, 70, 5)
    payload = torch.empty(hdr.payload_bytes, dtype=torch.uint8, device="cuda")
    kvg.kvg_int8_deposit(b.cache, b.seqs.block_tables[0], 0, 70, payload)
    ws = harness.artifact_workspace(hdr)
    kvg.kvg_artifact_seal(hdr, payload, ws)
    leaves = oracle_digest.leaf_digests(payload.cpu().numpy().tobytes(), 16 * 64)
    assert bytes(hdr.digest) == oracle_digest.merkle_root(leaves)
    path = str(tmp_path / "block")
    harness.save_artifact(path, hdr, payload)
    back, pinned = harness.load_artifact(path)
    assert kvg.kvg_artifact_verify(back, pinned, ws) == 0
    c, table = other_cache(kvg, b)
    kvg.kvg_int8_graft(c, back, pinned, table[0], 0, 5)
    again = torch.empty_like(payload)
    kvg.kvg_int8_deposit(c, table[0], 0, 70, again)
    assert torch.equal(payload, again)
    payload[-2] ^= 1                                            # of a scale
    assert kvg.kvg_artifact_verify(hdr, payload, ws) == -7


def test_graft_equals_fresh(kvg):  # noqa: F811
    """A prefix appended, deposited and grafted into another cache, a suffix and single tokens on top: the same bytes as where it
    was computed, whatever the pages, for a block that ends inside a page too."""
    heads, n = (8, 4, 128), 333
    fresh = Int8Batch([n], [0], heads, layers=2, seed=21, max_pages=32, spare_pages=9)
    rt, scale = kvg.rotary(), 1.0 / math.sqrt(128)
    rows = [fresh.rows(h) for h in (8, 4, 4)]
    kvg.kvg_int8_append(fresh.cache, fresh.seqs, fresh.packed, rt, None, 0, 2, *rows, torch.empty_like(rows[0]))
    hdr = kvg.kvg_int8_header_init(fresh.cache, n, int(fresh.start[0]))
    payload = torch.empty(hdr.payload_bytes, dtype=torch.uint8, device="cuda")
    kvg.kvg_int8_deposit(fresh.cache, fresh.seqs.block_tables[0], 0, n, payload)
    c, table = other_cache(kvg, fresh)
    kvg.kvg_int8_graft(c, hdr, payload, table[0], 0, int(fresh.start[0]))
    at = n
    for count in (35, 1, 1, 20, 1):
        q, k, v = (torch.randn(2, count, h, 128, generator=fresh.gen, device="cuda").to(torch.bfloat16) for h in (8, 4, 4))
        res = []
        for cache, tab in ((fresh.cache, fresh.seqs.block_tables), (c, table)):
            seqs = kvg.Seqs(tab, torch.tensor([at], dtype=torch.int32, device="cuda"), fresh.seqs.start_pos, at)
            packed = kvg.Packed(torch.tensor([0, count], dtype=torch.int32, device="cuda"), count, count)
            turned, out = torch.empty_like(q), torch.empty_like(q)
            kvg.kvg_int8_append(cache, seqs, packed, rt, None, 0, 2, q, k, v, turned)
            kvg.kvg_int8_attn(cache, seqs, packed, 0, 2, turned, scale, out, kvg.int8_attn_workspace(cache, seqs, packed, 2))
            res.append(out)
        assert torch.equal(bits(res[0]), bits(res[1]))
        at += count


def test_captured_steps_replay(kvg):  # noqa: F811
    """Two graphs, each an append and an attention of a step with workspaces of their own, replayed in turn with other lengths and eager work
    between: every replay against the eager calls on a copy."""
    b = Int8Batch([1, 1, 1], [20, 500, 31], (4, 2, 128), layers=2, seed=3, max_pages=40)
    q, k, v = b.rows(4), b.rows(2), b.rows(2)
    seqs = kvg.Seqs(b.seqs.block_tables, b.seqs.ctx_lens, b.seqs.start_pos, 600)
    rt = kvg.rotary()

    def step(cache, turned, out, ws):
        kvg.kvg_int8_append(cache, seqs, b.packed, rt, None, 0, 2, q, k, v, turned)
        kvg.kvg_int8_attn(cache, seqs, b.packed, 0, 2, turned, 0.09, out, ws)

    copy = kvg.Int8Cache(*(t.clone() for t in b.cache.tensors()), 4)
    buffers = [(torch.empty_like(q), torch.empty_like(q), kvg.int8_attn_workspace(b.cache, seqs, b.packed, 2)) for _ in range(3)]
    start = [t.clone() for t in b.cache.tensors()]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(b.cache, *buffers[i])
        graphs.append(g)
    for t, s in zip(b.cache.tensors(), start):
        assert torch.equal(bits(t), bits(s))                    # a capture runs nothing
    gen = torch.Generator(device="cuda").manual_seed(1)
    for turn in range(6):
        for x in (q, k, v):
            x.normal_(0.0, 1.0 + turn, generator=gen)
        b.seqs.ctx_lens.copy_(torch.tensor([20 + turn, 500 + turn, 31 + 90 * turn], dtype=torch.int32))
        graphs[turn % 2].replay()
        step(copy, *buffers[2])
        torch.cuda.synchronize()
        assert torch.equal(bits(buffers[turn % 2][1]), bits(buffers[2][1]))
        for t, s in zip(b.cache.tensors(), copy.tensors()):
            assert torch.equal(bits(t), bits(s))


def test_two_streams_at_once(kvg):  # noqa: F811
    b = Int8Batch([90, 1], [0, 2000], (8, 2, 128), seed=3)
    q = b.rows(8, 2.0)
    want = b.attend(q, 0.1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(want) for _ in range(2)]
    ws = [b.workspace() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, out, w in zip(streams, outs, ws):
            kvg.kvg_int8_attn(b.cache, b.seqs, b.packed, 0, 1, q, 0.1, out, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(bits(out), bits(want)) for out in outs)


def test_offsets_past_32_bits(kvg):  # noqa: F811
    """A layer of more than 2^31 bytes of integers: pages at its end."""
    heads = (1, 1, 256)
    n_pages = (1 << 31) // (16 * 256) + 40
    cache = kvg.Int8Cache.allocate(1, n_pages, *heads)
    table = torch.arange(n_pages - 20, n_pages, dtype=torch.int32, device="cuda")[None].contiguous()
    start = torch.zeros(1, dtype=torch.int64, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = 300
    q, k, v = (torch.randn(1, n, 1, 256, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    seqs = kvg.Seqs(table, torch.zeros(1, dtype=torch.int32, device="cuda"), start, 0)
    packed = kvg.Packed(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    small = kvg.Int8Cache.allocate(1, 20, *heads)
    res = []
    for c, t in ((cache, table), (small, (table - (n_pages - 20)).contiguous())):
        s = kvg.Seqs(t, seqs.ctx_lens, start, 0)
        kvg.kvg_int8_append(c, s, packed, kvg.rotary(), None, 0, 1, q, k, v, turned)
        kvg.kvg_int8_attn(c, s, packed, 0, 1, turned, 0.06, out, kvg.int8_attn_workspace(c, s, packed, 1))
        res.append(out.clone())
    assert torch.equal(bits(res[0]), bits(res[1])) and bool(torch.isfinite(host_norm(res[0])))


def host_norm(t):
    return t.float().norm()
