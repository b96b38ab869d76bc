"""Packed sequences as a serving program uses them: appended, attended, deposited, grafted into another cache and
continued there; captured into graphs; on other streams; with padded batches, loose bounds and large pools."""

import math

import numpy as np
import pytest
import torch

from tests.packed_helpers import TORCH, Batch, check_attention
from tests.test_gpu_packed import append, bits, make_rotary

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvg():
    from paper_2607_14431_amd import kvg as k
    return k


class Model:
    """A layer stack's calls over one cache: norm, rotation, append, attention, layer by layer."""

    def __init__(self, kvg, heads, dtype, layers, windows, n_pages, scaling="rotations"):
        self.kvg, self.heads, self.layers = kvg, heads, layers
        Hq, Hkv, D = heads
        self.cache = kvg.Cache.allocate(layers, n_pages, Hq, Hkv, D, TORCH[dtype], windows=windows)
        self.cache.k_pool.fill_(float("nan"))
        self.cache.v_pool.fill_(float("nan"))
        self.rt, self.theta = make_rotary(kvg, D, "half", D // 2, scaling, amplitude=1.2)
        gen = torch.Generator(device="cuda").manual_seed(77)
        raw = self.cache.raw_dtype
        self.norms = [kvg.HeadNorm(*(torch.randn(1, D, generator=gen, device="cuda").mul(0.2).to(raw) for _ in range(2)), 1e-6, 1.0)
                      for _ in range(layers)]
        self.scale = 1 / math.sqrt(D)

    def batch(self, table, ctxs, lens, pad=0, start=None, max_ctx=None, max_len=None):
        i32 = dict(dtype=torch.int32, device="cuda")
        cu = np.concatenate([[0], np.cumsum(lens)])
        seqs = self.kvg.Seqs(table, torch.tensor(ctxs, **i32), start if start is not None else
                             torch.zeros(len(lens), dtype=torch.int64, device="cuda"), max_ctx if max_ctx is not None else max(ctxs))
        return seqs, self.kvg.Packed(torch.tensor(cu, **i32), int(cu[-1]) + pad, max_len if max_len is not None else max(lens))

    def run(self, seqs, packed, rows, out, q=None, ws=None, stream=None):
        """rows: [layers][n_tokens][Hq + 2 Hkv][D], the projections' rows of every layer."""
        kvg, (Hq, Hkv, D) = self.kvg, self.heads
        q = torch.empty_like(out) if q is None else q
        ws = kvg.packed_attn_workspace(self.cache, seqs, packed, 1) if ws is None else ws
        for l in range(self.layers):
            x = rows[l:l + 1]
            kvg.kvg_norm_append(self.cache, seqs, packed, self.rt, self.norms[l], l, 1, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv],
                                x[:, :, Hq + Hkv:], q[l:l + 1], stream)
            kvg.kvg_packed_attn(self.cache, seqs, packed, l, 1, q[l:l + 1], self.scale, out[l:l + 1], ws, stream)
        return out


def token_rows(model, ids, seed):
    """The projections' rows of tokens `ids` (their values depend on the id alone): [layers][len][heads][D]."""
    Hq, Hkv, D = model.heads
    gen = torch.Generator().manual_seed(seed)
    every = torch.randn(model.layers, max(ids) + 1, Hq + 2 * Hkv, D, generator=gen) * 1.5
    return every[:, ids].to(device="cuda", dtype=model.cache.raw_dtype)


@pytest.mark.parametrize("dtype,heads,windows", [
    ("bf16", (4, 2, 256), None), ("bf16", (16, 2, 128), (0, 150)), ("fp8", (8, 4, 128), None), ("f32", (4, 2, 64), (70, 0))])
def test_deposit_graft_and_continue(kvg, dtype, heads, windows):
    """A block is filled by a packed call beside other sequences, deposited, grafted into another cache and continued
    there by a ragged batch (a suffix, single tokens): outputs and cache are byte for byte those of a fresh whole prompt."""
    Hq, Hkv, D = heads
    n_block, n_suffix, steps, layers = 600, 45, 3, 2
    n = n_block + n_suffix + steps
    pages = -(-n // 16)

    def model():
        return Model(kvg, heads, dtype, layers, windows, 3 * pages)

    rng = np.random.default_rng(3)
    fresh = model()
    table = torch.from_numpy(rng.permutation(3 * pages)[:pages].reshape(1, pages).astype(np.int32)).cuda()
    rows = token_rows(fresh, list(range(n)), 5)
    seqs, packed = fresh.batch(table, [0], [n])
    want = fresh.run(seqs, packed, rows, torch.empty(layers, n, Hq, D, dtype=rows.dtype, device="cuda"))
    assert want.float().isfinite().all()

    # the block, as the second of three sequences of one call
    store = model()
    lens = [17, n_block, 1]
    t3 = torch.from_numpy(rng.permutation(3 * pages).reshape(3, pages).astype(np.int32)).cuda()
    seqs, packed = store.batch(t3, [0, 0, 0], lens)
    other = token_rows(store, list(range(18)), 6)
    out = store.run(seqs, packed, torch.cat([other[:, :17], rows[:, :n_block], other[:, 17:]], 1),
                    torch.empty(layers, sum(lens), Hq, D, dtype=rows.dtype, device="cuda"))
    assert torch.equal(bits(out[:, 17:17 + n_block]), bits(want[:, :n_block]))
    rp = kvg.rope(10000.0, 0)
    hdr = kvg.kvg_artifact_header_init(store.cache, n_block, 0, rp)
    payload = torch.empty(hdr.payload_bytes, dtype=torch.uint8, device="cuda")
    kvg.kvg_deposit(store.cache, t3[1], 0, n_block, payload)

    # grafted at its own position, then the suffix beside a prompt and a single token, then single tokens
    here = model()
    t2 = torch.from_numpy(rng.permutation(3 * pages)[:2 * pages].reshape(2, pages).astype(np.int32)).cuda()
    kvg.kvg_graft(here.cache, hdr, payload, t2[1], 0, 0)
    at = n_block
    for lens in ([30, n_suffix], [1, 1], [0, 1], [1, 1]):
        ctx0 = {30: 0, 1: 30, 0: 31}[lens[0]]
        seqs, packed = here.batch(t2, [ctx0, at], lens)
        x = torch.cat([token_rows(here, list(range(40)), 6)[:, :lens[0]], rows[:, at:at + lens[1]]], 1)
        out = here.run(seqs, packed, x, torch.empty(layers, sum(lens), Hq, D, dtype=rows.dtype, device="cuda"))
        assert torch.equal(bits(out[:, lens[0]:]), bits(want[:, at:at + lens[1]])), (at, lens)
        at += lens[1]
    assert at == n
    both = []
    for m, row in ((fresh, table[0]), (here, t2[1])):
        p = torch.empty(kvg.kvg_payload_bytes(m.cache, n), dtype=torch.uint8, device="cuda")
        kvg.kvg_deposit(m.cache, row, 0, n, p)
        both.append(p)
    assert torch.equal(*both)


def test_single_tokens_beside_the_decode_call(kvg):
    """Plain rotary, no norm: the packed calls and kvg_decode_attn leave the same bytes in the cache."""
    heads, ctxs = (8, 4, 128), [0, 200, 1025]
    Hq, Hkv, D = heads
    a, b = (Batch([1, 1, 1], ctxs, heads, "bf16", layers=2, seed=31) for _ in range(2))
    q, k, v = a.rows(Hq, 2.0), a.rows(Hkv), a.rows(Hkv)
    qr, out = torch.empty_like(q), torch.empty_like(q)
    append(a, kvg.rotary(10000.0), None, q, k, v, qr)
    a.attend(qr, 0.1, out)
    dec = torch.empty(2, 3, Hq, D, device="cuda")
    rp = kvg.rope(10000.0)
    kvg.kvg_decode_attn(b.cache, b.seqs, rp, 0, 2, q, k, v, 0.1, dec, kvg.decode_workspace(b.cache, b.seqs, 2))
    assert torch.equal(bits(a.cache.k_pool), bits(b.cache.k_pool)) and torch.equal(bits(a.cache.v_pool), bits(b.cache.v_pool))
    check_attention(a, qr, out, 0.1)
    assert dec.isfinite().all()


@pytest.mark.parametrize("dtype,heads", [("bf16", (16, 8, 256)), ("fp8", (16, 2, 128)), ("bf16", (4, 2, 64)), ("f32", (4, 2, 64))])
def test_captured_steps(kvg, dtype, heads):
    """A mixed batch's append and attention of two layers, captured; the replays read what the tensors hold then, and a second
    graph that shares the workspace runs between them.  Every replay against the eager call."""
    Hq, Hkv, D = heads
    lens, ctxs, pages = [1, 90, 0, 1, 33], [700, 30, 5, 1300, 0], 90
    m = Model(kvg, heads, dtype, 2, (0, 200), 5 * pages)
    table = torch.randperm(5 * pages, device="cuda").to(torch.int32).view(5, pages)
    m.cache.k_pool.copy_(torch.randn(m.cache.k_pool.shape, device="cuda"))
    m.cache.v_pool.copy_(torch.randn(m.cache.v_pool.shape, device="cuda"))
    seqs, packed = m.batch(table, ctxs, lens, pad=3)
    inputs = [token_rows(m, list(range(packed.n_tokens)), 40 + i) for i in range(3)]
    eager = [m.run(seqs, packed, x, torch.full((2, packed.n_tokens, Hq, D), 7.0, dtype=x.dtype, device="cuda")).clone()
             for x in inputs]
    assert not torch.equal(eager[0], eager[1])
    graphs = []
    ws = kvg.packed_attn_workspace(m.cache, seqs, packed, 1)          # one for both: they never run at once
    for _ in range(2):
        rows, out = inputs[0].clone(), torch.full_like(eager[0], 7.0)
        q = torch.empty_like(out)
        m.run(seqs, packed, rows, out, q, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.run(seqs, packed, rows, out, q, ws)
        graphs.append((g, rows, out))
    for rep in range(4):
        for j, (g, rows, out) in enumerate(graphs):
            i = (rep + j) % 3
            rows.copy_(inputs[i])
            out.fill_(7.0)
            _ = torch.randn(1 << 18, device="cuda").sum()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits(out), bits(eager[i])), (rep, j)
    del graphs


def test_another_stream_and_two_calls_at_once(kvg):
    """Two batches on two streams at once, each with its own workspace; what they wait for was enqueued on their streams."""
    heads = (8, 4, 128)
    bs = [Batch([300, 1, 40], [900, 2000, 0], heads, "bf16", layers=2, seed=50 + i) for i in range(2)]
    qs = [b.rows(8, 2.0) for b in bs]
    want = [b.attend(q, 0.1) for b, q in zip(bs, qs)]
    streams = [torch.cuda.Stream() for _ in bs]
    outs = [torch.zeros_like(w) for w in want]
    spaces = [b.workspace() for b in bs]
    late = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b, q, l, o, w in zip(streams, bs, qs, late, outs, spaces):
            with torch.cuda.stream(s):
                l.copy_(q)
                b.attend(l, 0.1, o, w)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(bits(o), bits(w))
            o.zero_()
    b, s = bs[0], streams[1]                                     # a stream as an argument
    s.wait_stream(torch.cuda.current_stream())
    kvg.kvg_packed_attn(b.cache, b.seqs, b.packed, 0, 2, qs[0], 0.1, outs[0], spaces[0], s)
    s.synchronize()
    assert torch.equal(bits(outs[0]), bits(want[0]))


@pytest.mark.parametrize("dtype,heads,lens,ctxs", [
    ("bf16", (4, 2, 64), [300], [900]), ("bf16", (8, 2, 128), [130, 70], [800, 1100]), ("fp8", (4, 2, 256), [140], [1200]),
    ("f32", (4, 2, 64), [100], [900])])
@pytest.mark.parametrize("window", [0, 333])
def test_rows_do_not_depend_on_the_launch(kvg, dtype, heads, lens, ctxs, window):
    """A launch of one layer is split over segments, one of many layers is not: the same bytes for every layer."""
    L = 48
    one = Batch(lens, ctxs, heads, dtype, layers=1, windows=(window,), seed=60)
    q = one.rows(heads[0], 2.0)
    want = one.attend(q, 0.1)
    check_attention(one, q, want, 0.1, lambda n: range(0, n, 7))
    pools = [p.repeat(L, 1, 1, 1, 1) if p.dtype != torch.float8_e4m3fn else
             p.view(torch.uint8).repeat(L, 1, 1, 1, 1).view(p.dtype) for p in (one.cache.k_pool, one.cache.v_pool)]
    cache = kvg.Cache(pools[0], pools[1], heads[0], (window,) * L)
    out = torch.full((L, *want.shape[1:]), 7.0, dtype=want.dtype, device="cuda")
    small = kvg.kvg_packed_attn_workspace_bytes(one.cache, one.seqs, one.packed, 1)
    ws = kvg.packed_attn_workspace(cache, one.seqs, one.packed, L)
    if len(lens) == 1 and window == 0:
        assert small > ws.nbytes, "the one is meant to be split, the other not"
    kvg.kvg_packed_attn(cache, one.seqs, one.packed, 0, L, q.repeat(L, 1, 1, 1), 0.1, out, ws)
    for l in range(L):
        assert torch.equal(bits(out[l]), bits(want[0])), l


@pytest.mark.parametrize("dtype,heads,lens,ctxs", [
    ("bf16", (16, 2, 128), [1, 4, 1], [1500, 700, 3]), ("bf16", (4, 2, 256), [1], [1100]), ("fp8", (16, 8, 256), [16, 1], [600, 513]),
    ("bf16", (4, 2, 64), [2, 1], [1400, 511]), ("fp8", (4, 4, 128), [32, 1], [1000, 1023])])
@pytest.mark.parametrize("window", [0, 100, 700])
def test_few_rows_do_not_depend_on_the_launch(kvg, dtype, heads, lens, ctxs, window):
    """Workgroups of four waves in a small launch, of two in one of many layers: the same bytes for every layer."""
    L = 80
    one = Batch(lens, ctxs, heads, dtype, layers=1, windows=(window,), seed=61)
    q = one.rows(heads[0], 2.0)
    want = one.attend(q, 0.1)
    check_attention(one, q, want, 0.1)
    pools = [p.view(torch.uint8).repeat(L, 1, 1, 1, 1).view(p.dtype) for p in (one.cache.k_pool, one.cache.v_pool)]
    cache = kvg.Cache(pools[0], pools[1], heads[0], (window,) * L)
    out = torch.full((L, *want.shape[1:]), 7.0, dtype=want.dtype, device="cuda")
    kvg.kvg_packed_attn(cache, one.seqs, one.packed, 0, L, q.repeat(L, 1, 1, 1), 0.1, out,
                        kvg.packed_attn_workspace(cache, one.seqs, one.packed, L))
    for l in range(L):
        assert torch.equal(bits(out[l]), bits(want[0])), l


def test_loose_bounds_and_padding_change_nothing(kvg):
    """max_len, max_ctx_len and n_tokens are bounds: larger ones (a batch padded for a graph) give the same bytes."""
    b = Batch([1, 200, 9], [800, 100, 0], (8, 4, 128), "bf16", seed=70)
    rt, _ = make_rotary(kvg, 128)
    q, k, v = b.rows(8, 2.0), b.rows(4), b.rows(4)
    qo = torch.empty_like(q)
    append(b, rt, None, q, k, v, qo)
    want = b.attend(qo, 0.1)
    after = b.cache.k_pool.clone()
    for pad, max_len, max_ctx in ((50, 200, 800), (700, 201, 801), (0, 400, 400 + 16), (3000, 33, 800)):
        n = b.tokens + pad
        table = torch.cat([b.seqs.block_tables, torch.full((3, 64), -1, dtype=torch.int32, device="cuda")], 1)
        seqs = kvg.Seqs(table, b.seqs.ctx_lens, b.seqs.start_pos, max_ctx)
        packed = kvg.Packed(b.packed.cu_tokens, n, max_len)
        wide = [torch.full((1, n, *t.shape[2:]), float("nan"), dtype=t.dtype, device="cuda") for t in (q, k, v)]
        for w, t in zip(wide, (q, k, v)):
            w[:, :b.tokens] = t
        qp, op = (torch.full((1, n, 8, 128), 7.0, dtype=q.dtype, device="cuda") for _ in range(2))
        kvg.kvg_norm_append(b.cache, seqs, packed, rt, None, 0, 1, *wide, qp)
        kvg.kvg_packed_attn(b.cache, seqs, packed, 0, 1, qp, 0.1, op, kvg.packed_attn_workspace(b.cache, seqs, packed, 1))
        keep = [s for s in range(3) if b.lens[s] <= max_len and b.ctxs[s] <= max_ctx]
        assert len(keep) >= 2
        for s in range(3):
            r = slice(int(b.cu[s]), int(b.cu[s + 1]))
            if s in keep:
                assert torch.equal(bits(qp[:, r]), bits(qo[:, r])) and torch.equal(bits(op[:, r]), bits(want[:, r])), (pad, s)
            else:
                assert bool((qp[:, r] == 7.0).all()) and bool((op[:, r] == 7.0).all()), (pad, s)
        assert bool((qp[:, b.tokens:] == 7.0).all()) and bool((op[:, b.tokens:] == 7.0).all())
        assert torch.equal(bits(b.cache.k_pool), bits(after))


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 4, 128)), ("fp8", (8, 4, 256)), ("f32", (4, 2, 64))])
def test_pools_and_rows_past_32_bits(kvg, dtype, heads):
    """Pages whose bytes and elements lie past 2^32 and 2^31, packed rows past 2^31 elements: the bytes of small ones."""
    Hq, Hkv, D = heads
    lens, ctxs = [40, 1], [600, 90]
    b = Batch(lens, ctxs, heads, dtype, layers=1, seed=80)
    rt, _ = make_rotary(kvg, D)
    q, k, v = b.rows(Hq, 2.0), b.rows(Hkv), b.rows(Hkv)
    qo = torch.empty_like(q)
    append(b, rt, None, q, k, v, qo)
    want = b.attend(qo, 0.1)
    used = torch.from_numpy(b.table.reshape(-1).astype(np.int64)).cuda()
    page = Hkv * 16 * D
    n_pages = (1 << 32) // page + len(used) + 5
    shift = n_pages - b.cache.n_pages
    pools = []
    for p in (b.cache.k_pool, b.cache.v_pool):
        big = torch.empty((1, n_pages, Hkv, 16, D), dtype=p.dtype, device="cuda")
        bits(big[:, shift:]).copy_(bits(p))
        pools.append(big)
    cache = kvg.Cache(pools[0], pools[1], Hq)
    seqs = kvg.Seqs(b.seqs.block_tables + shift, b.seqs.ctx_lens, b.seqs.start_pos, max(ctxs))
    lead = (1 << 31) // (Hq * D)
    n = lead + b.tokens
    packed = kvg.Packed(b.packed.cu_tokens + lead, n, max(lens))
    def far(t, heads):
        x = torch.empty((1, n, heads, D), dtype=t.dtype, device="cuda")
        x[:, lead:] = t
        return x
    kf, vf = far(k, Hkv), far(v, Hkv)
    q_far, qo_far = far(q, Hq), torch.empty((1, n, Hq, D), dtype=q.dtype, device="cuda")
    kvg.kvg_norm_append(cache, seqs, packed, rt, None, 0, 1, q_far, kf, vf, qo_far)
    assert torch.equal(bits(qo_far[:, lead:]), bits(qo))
    for big, p in zip(pools, (b.cache.k_pool, b.cache.v_pool)):
        assert torch.equal(bits(big[:, shift:]), bits(p))
    del kf, vf, q_far
    out = torch.empty_like(qo_far)
    kvg.kvg_packed_attn(cache, seqs, packed, 0, 1, qo_far, 0.1, out, kvg.packed_attn_workspace(cache, seqs, packed, 1))
    assert torch.equal(bits(out[:, lead:]), bits(want))
    pos = torch.arange(n, device="cuda")
    if dtype != "fp8":
        y, z = torch.empty_like(out), torch.empty_like(q)
        kvg.kvg_rotate(rt, pos, qo_far[0], y[0])
        kvg.kvg_rotate(rt, pos[lead:], qo[0], z[0])
        assert torch.equal(bits(y[0, lead:]), bits(z[0]))


def test_workspace_of_one_byte_less_is_refused(kvg):
    b = Batch([100, 1], [2000, 2000], (8, 4, 128), "bf16", seed=90)
    q = b.rows(8)
    n = kvg.kvg_packed_attn_workspace_bytes(b.cache, b.seqs, b.packed, 1)
    ws = torch.full((n + 256,), 99, dtype=torch.uint8, device="cuda")
    b.attend(q, 0.1, ws=ws[:n])
    torch.cuda.synchronize()
    assert bool((ws[n:] == 99).all())                            # nothing past it is written
    with pytest.raises(kvg.KvgError):
        b.attend(q, 0.1, ws=ws[:n - 1])


def test_same_page_in_two_tables(kvg):
    """Sequences that share a prefix's pages (as a graft into shared pages leaves them) read them alike."""
    b = Batch([20, 35, 1], [640, 640, 640], (8, 2, 128), "bf16", seed=91)
    shared = b.table.copy()
    shared[1, :40] = shared[0, :40]
    shared[2, :40] = shared[0, :40]
    b.table = shared
    b.seqs.block_tables.copy_(torch.from_numpy(shared))
    q = b.rows(8, 2.0)
    check_attention(b, q, b.attend(q, 0.1), 0.1)


def test_workspace_covers_any_layers(kvg):
    """The size is asked for without the first layer: it serves every one, where windows change how a launch is split."""
    b = Batch([700, 1, 60], [900, 2500, 30], (8, 2, 128), "bf16", layers=6, windows=(0, 128, 128, 200, 0, 0), seed=92)
    q = b.rows(8, 2.0)
    want = b.attend(q, 0.1)
    for n in (1, 2, 3, 6):
        size = kvg.kvg_packed_attn_workspace_bytes(b.cache, b.seqs, b.packed, n)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        for l0 in range(6 - n + 1):
            out = torch.empty_like(want[l0:l0 + n])
            kvg.kvg_packed_attn(b.cache, b.seqs, b.packed, l0, n, q[l0:l0 + n], 0.1, out, ws)
            rows = torch.from_numpy(np.concatenate([np.arange(b.cu[s], b.cu[s + 1]) for s in range(3)]).astype(np.int64)).cuda()
            assert torch.equal(bits(out[:, rows]), bits(want[l0:l0 + n][:, rows])), (n, l0)


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 4, 128)), ("fp8", (4, 2, 256)), ("f32", (4, 2, 64))])
def test_a_graph_replays_with_other_lengths(kvg, dtype, heads):
    """The lengths are the device's: a graph captured for its bounds serves every batch within them."""
    Hq, Hkv, D = heads
    B, rows_max, max_len, max_ctx, pages = 4, 140, 100, 1400, 95
    m = Model(kvg, heads, dtype, 1, None, B * pages)
    for pool in (m.cache.k_pool, m.cache.v_pool):
        pool.copy_(torch.randn(pool.shape, device="cuda"))
    table = torch.randperm(B * pages, device="cuda").to(torch.int32).view(B, pages)
    i32 = dict(dtype=torch.int32, device="cuda")
    cu, ctx, start = torch.zeros(B + 1, **i32), torch.zeros(B, **i32), torch.zeros(B, dtype=torch.int64, device="cuda")
    seqs, packed = kvg.Seqs(table, ctx, start, max_ctx), kvg.Packed(cu, rows_max, max_len)
    rows = token_rows(m, list(range(rows_max)), 9)
    out, q = (torch.full((1, rows_max, Hq, D), 7.0, dtype=rows.dtype, device="cuda") for _ in range(2))
    ws = kvg.packed_attn_workspace(m.cache, seqs, packed, 1)
    m.run(seqs, packed, rows, out, q, ws)                        # nothing to do: all lengths are 0
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((q == 7.0).all())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        m.run(seqs, packed, rows, out, q, ws)
    for lens, ctxs, st in (([1, 1, 1, 1], [1400, 3, 0, 700], [0, 5, 9, 2]), ([100, 0, 33, 7], [0, 9, 1300, 511], [1, 1, 1, 1]),
                           ([0, 0, 0, 1], [0, 0, 0, 0], [0, 0, 0, 3]), ([40, 60, 1, 39], [1000, 1400, 64, 0], [7, 0, 0, 0])):
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)))
        ctx.copy_(torch.tensor(ctxs, dtype=torch.int32))
        start.copy_(torch.tensor(st))
        want, wq = torch.full_like(out, 7.0), torch.full_like(q, 7.0)
        m.run(seqs, packed, rows, want, wq)
        for _ in range(2):
            out.fill_(7.0)
            q.fill_(7.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits(out), bits(want)) and torch.equal(bits(q), bits(wq)), lens
        assert bool((out[:, sum(lens):] == 7.0).all()) and out[:, :sum(lens)].float().isfinite().all()
    del g


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 4, 128)), ("bf16", (16, 2, 64)), ("fp8", (4, 2, 256)), ("f32", (4, 2, 64))])
def test_a_query_that_is_not_finite_keeps_to_its_row(dtype, heads):
    b = Batch([70, 3, 1], [600, 40, 1000], heads, dtype, seed=95)
    q = b.rows(heads[0], 2.0)
    want = b.attend(q, 0.1)
    bad = [(0, 1, 3), (69, 0, 0), (71, heads[0] - 1, 5), (73, 2, 7)]
    for t, h, x in bad:
        q[0, t, h, x] = float("nan") if t % 2 else float("inf")
    got = b.attend(q, 0.1)
    for t, h, _ in bad:
        assert got[0, t, h].isnan().all(), (t, h)
        got[0, t, h] = want[0, t, h]
    assert torch.equal(bits(got), bits(want))
