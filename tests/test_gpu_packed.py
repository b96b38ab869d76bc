"""Packed sequences on the GPU: rotary positions, norms with append, attention, against the oracle in fp64, at the lengths,
masks, strides and metadata where they can go wrong."""

import math

import numpy as np
import pytest
import torch

from oracle import packed as oracle
from tests.packed_helpers import HALF_STEP, TORCH, U, Batch, check_attention, host

pytestmark = pytest.mark.gpu

SCALED = dict(factor=6.0, original_len=3000.0, fast=20.0, slow=1.5)
SCALINGS = ["plain", "linear", "base", "rotations", "index"]
PAIRINGS = ["half", "interleaved"]


@pytest.fixture(scope="module")
def kvg():
    from paper_2607_14431_amd import kvg as k
    return k


def make_rotary(kvg, head_dim, pairing="half", dim=0, scaling="plain", base=10000.0, amplitude=1.0):
    rt = kvg.rotary(base, PAIRINGS.index(pairing), dim, SCALINGS.index(scaling), amplitude=amplitude, **SCALED)
    theta = oracle.frequencies(dim or head_dim, base, scaling, **SCALED)
    return rt, theta


def pair_size(x, dim, pairing):
    """sqrt(a^2 + b^2) of each value's pair (its own size past the rotated part)."""
    ia, ib = oracle.pair_index(dim, pairing)
    r = np.abs(x).copy()
    r[..., ia] = r[..., ib] = np.hypot(x[..., ia], x[..., ib])
    return r


def rotated_bound(want, size, dtype, rel=0.0):
    """An fp32 rotation of values of pair size `size`, known to rel, and one rounding: cos and sin are rounded (u each of
    their share of the pair: sqrt 2 u), a product and the sum round once each (2 u), the angle's fp64 error is far below."""
    off = (4 * U + rel * 1.5) * size
    return off + HALF_STEP[dtype] * (np.abs(want) + off) + (2.0 ** -10 if dtype == "fp8" else 1e-38)


# ---------------------------------------------------------------------------- rotary positions

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing", PAIRINGS)
@pytest.mark.parametrize("head_dim,dim,scaling,tokens,heads", [
    (64, 0, "plain", 1, 1), (128, 64, "index", 37, 5), (256, 0, "rotations", 3, 24), (256, 48, "base", 19, 2),
    (64, 16, "linear", 130, 3)])
def test_rotate(kvg, dtype, pairing, head_dim, dim, scaling, tokens, heads):
    rt, theta = make_rotary(kvg, head_dim, pairing, dim, scaling, amplitude=1.25)
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.randn(tokens, heads + 3, head_dim, generator=gen, device="cuda").to(TORCH[dtype])
    x = wide[:, 1:1 + heads]
    pos = torch.randint(-100, 3_000_000, (tokens,), generator=gen, device="cuda")
    pos[0] = 0
    y = torch.full((tokens, heads, head_dim), 7.0, dtype=TORCH[dtype], device="cuda")
    kvg.kvg_rotate(rt, pos, x, y)
    want = oracle.rotate(host(x), pos.cpu().numpy(), theta, pairing, 1.25)
    size = 1.25 * pair_size(host(x), 2 * len(theta), pairing)
    assert np.all(np.abs(host(y) - want) <= rotated_bound(want, size, dtype))
    assert torch.equal(y[..., 2 * len(theta):], x[..., 2 * len(theta):])          # left as they are
    before = wide.clone()
    kvg.kvg_rotate(rt, pos, x, x)                                                  # in place, strided
    assert torch.equal(x, y)
    assert torch.equal(wide[:, :1], before[:, :1]) and torch.equal(wide[:, 1 + heads:], before[:, 1 + heads:])


def test_rotate_by_minus_positions_undoes_it(kvg):
    rt, _ = make_rotary(kvg, 128, "half", 96, "rotations")
    x = torch.randn(50, 4, 128, device="cuda")
    pos = torch.arange(50, device="cuda") * 4099
    y, z = torch.empty_like(x), torch.empty_like(x)
    kvg.kvg_rotate(rt, pos, x, y)
    kvg.kvg_rotate(rt, -pos, y, z)
    size = pair_size(host(x), 96, "half")
    assert np.all(np.abs(host(z) - host(x)) <= 2 * rotated_bound(host(x), size, "f32"))


def test_rotate_keeps_inf_and_nan_to_their_pairs(kvg):
    rt, _ = make_rotary(kvg, 64, "interleaved", 32)
    x = torch.randn(4, 2, 64, device="cuda").to(torch.bfloat16)
    clean = torch.empty_like(x)
    pos = torch.tensor([5, 6, 7, 8], device="cuda")
    kvg.kvg_rotate(rt, pos, x, clean)
    x[1, 0, 6], x[2, 1, 40] = float("nan"), float("inf")
    y = torch.empty_like(x)
    kvg.kvg_rotate(rt, pos, x, y)
    assert y[1, 0, 6:8].isnan().all() and y[2, 1, 40].isinf()
    clean[1, 0, 6:8], clean[2, 1, 40] = y[1, 0, 6:8], y[2, 1, 40]
    assert torch.equal(y.view(torch.int16), clean.view(torch.int16))


# ---------------------------------------------------------------------------- norms, rotation, append

def append(batch, rt, norm, q, k, v, out):
    batch.kvg.kvg_norm_append(batch.cache, batch.seqs, batch.packed, rt, norm, 0, batch.layers, q, k, v, out)


def bits(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("heads,pairing,dim,scaling,wide", [
    ((4, 2, 64), "half", 0, "plain", 0), ((8, 8, 128), "interleaved", 64, "index", 6), ((16, 2, 256), "half", 128, "rotations", 4),
    ((8, 4, 64), "half", 16, "base", 2), ((1, 1, 256), "interleaved", 0, "linear", 0)])
def test_norm_append(kvg, dtype, heads, pairing, dim, scaling, wide):
    Hq, Hkv, D = heads
    b = Batch([3, 0, 1, 40, 17], [0, 5, 31, 16, 250], heads, dtype, layers=2, seed=5, lead=2, tail=3, poison=3.0)
    rt, theta = make_rotary(kvg, D, pairing, dim, scaling, amplitude=1.1)
    q, k, v = b.rows(Hq, 1.5, wide), b.rows(Hkv, 1.5, wide), b.rows(Hkv, 1.5, wide)
    qw, kw = (torch.randn(2, D, generator=b.gen, device="cuda").mul(0.2).to(TORCH[b.raw]) for _ in range(2))
    norm = kvg.HeadNorm(qw, kw, 1e-6, 1.0)
    before = b.cache.k_pool.clone(), b.cache.v_pool.clone()
    out = torch.full((2, b.tokens, Hq, D), 7.0, dtype=TORCH[b.raw], device="cuda")
    append(b, rt, norm, q, k, v, out)
    # the norm's factor: a sum of D squares in runs of 8 and a tree (u of it each: at most 8 + 6 roundings), halved by the
    # root; mean, eps, root, quotient, product, weight sum and product round once each
    rel = (14 / 2 + 7) * U
    expect = [before[0].clone(), before[1].clone()]
    for l in range(2):
        for s, n in enumerate(b.lens):
            if n == 0:
                continue
            r = slice(int(b.cu[s]), int(b.cu[s]) + n)
            pos = b.start[s] + b.ctxs[s] + np.arange(n)
            for src, w, dst in ((q, qw, None), (k, kw, 0)):
                x = oracle.rms_norm(host(src[l, r]), host(w[l]), 1e-6, 1.0)
                want = oracle.rotate(x, pos, theta, pairing, 1.1)
                size = 1.1 * pair_size(x, 2 * len(theta), pairing)
                if dst is None:
                    got, dt = host(out[l, r]), b.raw
                else:
                    got, dt = b.keys_values(l, s)[0][b.ctxs[s]:], dtype
                bad = np.abs(got - want) > rotated_bound(want, size, dt, rel)
                assert not bad.any(), (l, s, "q" if dst is None else "k", np.argwhere(bad)[0])
            for i in range(n):                                   # values: the bytes torch stores, in the tokens' rows
                t = b.ctxs[s] + i
                page = int(b.table[s, t // 16])
                expect[0][l, page, :, t % 16] = b.cache.k_pool[l, page, :, t % 16]
                expect[1][l, page, :, t % 16] = v[l, r][i].to(TORCH[dtype])
    for got, want in zip((b.cache.k_pool, b.cache.v_pool), expect):
        assert torch.equal(bits(got), bits(want)), "other cache rows changed, or values differ"
    rest = torch.from_numpy(b.outside()).cuda()
    assert len(rest) == 5 and bool((out[:, rest] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("pairing", [0, 1])
def test_plain_append_gives_the_bytes_of_kvg_append(kvg, dtype, pairing):
    for D in (64, 256):
        a, c = (Batch([21, 21], [7, 40], (4, 2, D), dtype, layers=3, seed=9, poison=3.0) for _ in range(2))
        k, v = a.rows(2), a.rows(2)
        append(a, kvg.rotary(10000.0, pairing), None, None, k, v, None)
        kk, vv = (x.view(3, 2, 21, 2, D) for x in (k, v))
        kvg.kvg_append(c.cache, c.seqs, kvg.rope(10000.0, pairing), 0, 3, 21, kk, vv)
        assert torch.equal(bits(a.cache.k_pool), bits(c.cache.k_pool)) and torch.equal(bits(a.cache.v_pool), bits(c.cache.v_pool))


def test_append_queries_in_place_and_zero_rows(kvg):
    b = Batch([5, 9], [3, 0], (8, 2, 128), "bf16", seed=2, poison=3.0)
    rt, _ = make_rotary(kvg, 128)
    w = torch.ones(1, 128, dtype=torch.bfloat16, device="cuda")
    q, k, v = b.rows(8), b.rows(2), b.rows(2)
    q[0, 4, 3] = 0.0                                             # a zero head stays zero (eps in the root)
    out = torch.empty_like(q)
    append(b, rt, kvg.HeadNorm(w, None, 1e-6), q, k, v, out)
    assert bool((out[0, 4, 3] == 0).all())
    append(b, rt, kvg.HeadNorm(w, None, 1e-6), q, k, v, q)
    assert torch.equal(q, out)


def test_append_skips_bad_metadata_and_pages(kvg):
    """Sequences whose metadata is not as demanded, and pages outside the pool, are skipped; the others are as ever."""
    rt, _ = make_rotary(kvg, 64)
    def fresh():
        b = Batch([4, 5, 6, 7], [0, 16, 3, 40], (4, 2, 64), "bf16", seed=4, poison=3.0)
        return b, b.rows(4), b.rows(2), b.rows(2)
    good, q, k, v = fresh()
    want = torch.full_like(q, 7.0)
    append(good, rt, None, q, k, v, want)
    for what in ("ctx", "cu", "page", "len", "negative"):
        b, q, k, v = fresh()
        out = torch.full_like(q, 7.0)
        pages = b.cache.k_pool.clone()
        bad = 1
        if what == "ctx":
            b.seqs.ctx_lens[1] = 41                             # above max_ctx_len
        elif what == "negative":
            b.seqs.ctx_lens[1] = -1
        elif what == "cu":                                      # sequence 3 ends past the rows
            b.packed.cu_tokens[4] = b.tokens + 9
            bad = 3
        elif what == "len":                                     # longer than max_len: sequences 1 and 2 merge into 1
            b.packed.cu_tokens[2] = b.packed.cu_tokens[3]
        else:
            b.seqs.block_tables[1, 1] = 1 << 30
        append(b, rt, None, q, k, v, out)
        for s in range(4):
            r = slice(int(b.cu[s]), int(b.cu[s + 1]))
            if what == "len" and s == 2:
                continue
            if s != bad or what == "page":
                assert torch.equal(out[:, r], want[:, r]), (what, s)
            else:
                assert bool((out[:, r] == 7.0).all()), (what, s)
        for s in range(4):
            if s == bad or (what == "len" and s == 2):
                p = torch.from_numpy(b.table[s].astype(np.int64)).cuda()
                assert torch.equal(b.cache.k_pool[:, p].view(torch.int16), pages[:, p].view(torch.int16)), (what, s)


# ---------------------------------------------------------------------------- attention

GEOMETRY = [(2, 2, 64), (4, 2, 128), (8, 2, 64), (16, 2, 128), (2, 1, 256), (8, 1, 256), (4, 4, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("heads", GEOMETRY, ids=lambda h: "x".join(map(str, h)))
def test_attention_lengths(dtype, heads):
    """One token, none, odd lengths around 16, 32, 64 and 512 keys, with and without cached tokens."""
    b = Batch([1, 0, 33, 2, 64, 65, 7, 1, 130], [0, 9, 0, 15, 448, 447, 511, 1023, 1], heads, dtype, seed=11, lead=1, tail=2)
    q = b.rows(heads[0], 2.0, wide=4)
    out = b.attend(q, 1 / math.sqrt(heads[2]))
    check_attention(b, q, out, 1 / math.sqrt(heads[2]))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
def test_attention_single_tokens(dtype):
    """A decode step: every sequence one token, contexts of nothing to thousands."""
    for heads in ((16, 8, 256), (16, 2, 128), (4, 2, 64)):
        b = Batch([1] * 6, [0, 1, 63, 512, 1500, 2047], heads, dtype, layers=2, seed=12)
        q = b.rows(heads[0], 2.0)
        check_attention(b, q, b.attend(q, 1 / math.sqrt(heads[2])), 1 / math.sqrt(heads[2]))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("windows", [(1, 0), (16, 70), (600, 512), (64, 5000)])
def test_attention_windows(dtype, windows):
    b = Batch([1, 200, 37, 1], [900, 0, 555, 40], (4, 2, 128), dtype, layers=2, windows=windows, seed=13)
    q = b.rows(4, 2.0)
    check_attention(b, q, b.attend(q, 0.09), 0.09)


@pytest.mark.parametrize("dtype,heads", [("bf16", (8, 4, 128)), ("bf16", (4, 2, 256)), ("fp8", (4, 2, 128)), ("f32", (4, 2, 64))])
def test_attention_long_prompt(dtype, heads):
    """Prompts of several thousand tokens: rows at the ends, around the tile edges, and in the middle."""
    b = Batch([2500, 1, 700], [0, 3000, 1200], heads, dtype, seed=14)
    q = b.rows(heads[0], 2.0)
    scale = 1 / math.sqrt(heads[2])
    pick = lambda n: [0, 1, 31, 32, 63, 64, 127, 128, 255, 256, 511, 512, 513, 1023, 1024, n // 2, n - 2, n - 1]  # noqa: E731
    check_attention(b, q, b.attend(q, scale), scale, pick)


def test_attention_peaked_scores():
    """Scores of std 8 and needles: weights concentrate on few keys, references move late."""
    b = Batch([90, 1], [700, 1400], (4, 2, 128), "bf16", seed=15, k_sigma=2.0)
    q = b.rows(4, 4.0)
    out = b.attend(q, 1 / math.sqrt(128))
    check_attention(b, q, out, 1 / math.sqrt(128))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (16, 2, 128), (4, 2, 256)], ids=lambda h: "x".join(map(str, h)))
@pytest.mark.parametrize("windows", [None, (300,)], ids=["full", "window"])
def test_rows_do_not_depend_on_cuts_or_neighbours(dtype, heads, windows):
    """A prompt in one call, in ragged pieces, a token at a time at its end, alone and among other sequences: the same
    bytes for every row."""
    n, Hq = 1400, heads[0]
    whole = Batch([n], [0], heads, dtype, windows=windows, seed=16)
    q = whole.rows(Hq, 2.0)
    scale = 1 / math.sqrt(heads[2])
    want = whole.attend(q, scale)
    kvg = whole.kvg

    def piece(t0, t1, extra):
        """Rows [t0, t1) as the middle sequence of a batch with `extra` others."""
        ctxs = [3 * e for e in range(extra)] + [t0]
        lens = [2 + 31 * e for e in range(extra)] + [t1 - t0]
        pool_k, pool_v = whole.cache.k_pool, whole.cache.v_pool
        table = torch.from_numpy(np.repeat(whole.table, extra + 1, axis=0)).cuda()
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        rows = torch.randn(1, int(cu[-1]), Hq, heads[2], device="cuda").to(q.dtype)
        rows[:, int(cu[-2]):] = q[:, t0:t1]
        seqs = kvg.Seqs(table, torch.tensor(ctxs, dtype=torch.int32, device="cuda"),
                        torch.zeros(extra + 1, dtype=torch.int64, device="cuda"), max(ctxs))
        packed = kvg.Packed(torch.from_numpy(cu).cuda(), int(cu[-1]), max(lens))
        cache = kvg.Cache(pool_k, pool_v, Hq, windows)
        out = torch.empty_like(rows)
        kvg.kvg_packed_attn(cache, seqs, packed, 0, 1, rows, scale, out, kvg.packed_attn_workspace(cache, seqs, packed, 1))
        return out[:, int(cu[-2]):]

    for t0, t1, extra in ((0, 700, 0), (700, 701, 0), (701, 1400, 2), (5, 40, 1), (1399, 1400, 0), (1390, 1400, 3), (512, 600, 0),
                          (0, 1, 2), (1000, 1024, 1)):
        got = piece(t0, t1, extra)
        assert torch.equal(bits(got), bits(want[:, t0:t1])), (t0, t1, extra)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (2, 1, 256)], ids=lambda h: "x".join(map(str, h)))
def test_inf_and_nan_stay_with_the_rows_that_see_them(dtype, bad, heads):
    """A value (and a key) at token 70 that is not finite: rows before it, and rows whose window has passed it, keep
    their bytes; the rows that see a NaN value are NaN in that dimension."""
    n, W = 200, 60
    for which in ("v", "k"):
        for windows in (None, (W,)):
            b = Batch([n, 3], [10, 100], heads, dtype, windows=windows, seed=17)
            q = b.rows(heads[0], 2.0)
            scale = 1 / math.sqrt(heads[2])
            want = b.attend(q, scale)
            pool = b.cache.v_pool if which == "v" else b.cache.k_pool
            pool[0, int(b.table[0, 70 // 16]), 0, 70 % 16, 5] = bad
            got = b.attend(q, scale)
            index = 10 + np.arange(n)
            seen = (index >= 70) & ((index < 70 + W) if windows else True)
            group = heads[0] // heads[1]
            keep = torch.ones_like(got, dtype=torch.bool)
            keep[:, torch.from_numpy(np.flatnonzero(seen)).cuda(), :group] = False
            assert torch.equal(bits(got)[keep], bits(want)[keep]), (which, windows)
            hit = got[0, torch.from_numpy(np.flatnonzero(seen)).cuda()][:, :group, 5]
            if which == "v" and math.isnan(bad):
                assert hit.isnan().all()
            elif which == "v":
                assert not hit.isfinite().any()


@pytest.mark.parametrize("dtype,heads,lens,ctxs", [
    ("bf16", (4, 2, 64), [40, 3], [0, 20]), ("bf16", (2, 1, 256), [6, 60], [30, 0]), ("f32", (4, 2, 128), [50], [3]),
    ("bf16", (16, 8, 128), [1] * 40, [20] * 40), ("bf16", (8, 2, 128), [200], [500])])
def test_infinities_of_both_signs(dtype, heads, lens, ctxs):
    """In one dimension a value is +Inf, two tokens later another -Inf: rows that see the first alone are +Inf there, rows that
    see both are NaN, the same in every call.  Single tokens go in either kernel, by the batch."""
    b = Batch(lens, ctxs, heads, dtype, seed=20)
    q = b.rows(heads[0], 1.0)
    scale = 0.5 / math.sqrt(heads[2])
    want = b.attend(q, scale)
    for s, (n, c) in enumerate(zip(lens, ctxs)):
        first = c + n // 3                                       # some rows see neither
        for t, v in ((first, math.inf), (first + 2, -math.inf)):
            if t < c + n:
                b.cache.v_pool[0, int(b.table[s, t // 16]), :, t % 16, 7] = v
    got = b.attend(q, scale)
    for s, (n, c) in enumerate(zip(lens, ctxs)):
        first = c + n // 3
        for i in range(n):
            row, old = got[0, int(b.cu[s]) + i].clone(), want[0, int(b.cu[s]) + i]
            if c + i >= first + 2:
                assert row[:, 7].isnan().all(), (s, i)
            elif c + i >= first:
                assert (row[:, 7] == math.inf).all(), (s, i)
            else:
                assert torch.equal(row[:, 7], old[:, 7]), (s, i)
            row[:, 7] = old[:, 7]
            assert torch.equal(row, old), (s, i)
    for _ in range(3):
        assert torch.equal(bits(b.attend(q, scale)), bits(got))


def test_attention_skips_bad_metadata():
    for what in ("ctx", "negative", "cu", "order", "page"):
        b = Batch([4, 50, 6, 70], [0, 16, 3, 600], (4, 2, 64), "bf16", seed=18)
        q = b.rows(4, 2.0)
        want = b.attend(q, 0.125)
        bad = [1]
        if what == "ctx":
            b.seqs.ctx_lens[1] = 601
        elif what == "negative":
            b.seqs.ctx_lens[1] = -5
        elif what == "cu":
            b.packed.cu_tokens[4] = b.tokens + 1
            bad = [3]
        elif what == "order":                                   # descends: sequence 1 gone, sequence 2 too long
            b.packed.cu_tokens[2] = -3
            bad = [1, 2]
        else:
            b.seqs.block_tables[1, 1] = -7                      # unspecified values, no fault
        got = b.attend(q, 0.125)
        for s in range(4):
            r = slice(int(b.cu[s]), int(b.cu[s + 1]))
            if s not in bad:
                assert torch.equal(got[:, r], want[:, r]), (what, s)
            elif what != "page":
                assert bool((got[:, r] == 7.0).all()), (what, s)


def test_many_sequences():
    """More sequences than a wave has lanes, most of them single tokens or empty."""
    rng = np.random.default_rng(19)
    lens = [int(x) for x in rng.choice([0, 1, 1, 1, 5, 40], 150)]
    ctxs = [int(x) for x in rng.integers(0, 90, 150)]
    b = Batch(lens, ctxs, (4, 2, 64), "bf16", seed=19)
    rt, theta = make_rotary(b.kvg, 64)
    q, k, v = b.rows(4, 2.0), b.rows(2), b.rows(2)
    out = torch.full_like(q, 7.0)
    append(b, rt, None, q, k, v, out)
    for s in (0, 63, 64, 65, 128, 149):
        r = slice(int(b.cu[s]), int(b.cu[s + 1]))
        want = oracle.rotate(host(q[0, r]), b.start[s] + ctxs[s] + np.arange(lens[s]), theta, "half")
        assert np.all(np.abs(host(out[0, r]) - want) <= rotated_bound(want, pair_size(host(q[0, r]), 64, "half"), "bf16"))
    check_attention(b, out, b.attend(out, 0.125), 0.125)
