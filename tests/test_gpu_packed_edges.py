"""Packed sequences on the GPU at the edges of what their calls allow: blocks of scaled rotaries relocated, values that are not
finite, and single-segment batches of few rows."""

import math

import numpy as np
import pytest
import torch

from oracle import packed as oracle
from tests.packed_helpers import U, Batch, attention_bound, check_attention, host
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


# ---------------------------------------------------------------------------- values fp8 cannot hold

@pytest.mark.parametrize("call", ["packed", "packed, normed", "append", "decode"])
@pytest.mark.parametrize("pairing", [0, 1])
def test_fp8_caches_saturate_and_keep_nan(kvg, call, pairing):
    """Values beyond +-448 and infinities are stored as +-448, NaN as NaN (in a key: in its pair; in a normed one: in its
    head); everything else is stored as ever."""
    B, D = 3, 64
    n = 1 if call == "decode" else 4
    fresh = lambda: Batch([n] * B, [0, 20, 5], (4, 2, D), "fp8", seed=23, poison=3.0)  # noqa: E731
    weight = torch.ones(1, D, dtype=torch.bfloat16, device="cuda")

    def stored(b, k, v):
        if call.startswith("packed"):
            append(b, kvg.rotary(10000.0, pairing), None if call == "packed" else kvg.HeadNorm(None, weight, 1e-6), None, k, v, None)
        else:
            kk, vv = (x.view(1, B, n, 2, D) for x in (k, v))
            if call == "append":
                kvg.kvg_append(b.cache, b.seqs, kvg.rope(10000.0, pairing), 0, 1, n, kk, vv)
            else:
                out = torch.empty(1, B, 4, D, device="cuda")
                kvg.kvg_decode_attn(b.cache, b.seqs, kvg.rope(10000.0, pairing), 0, 1, b.rows(4).view(1, B, 4, D), kk[:, :, 0],
                                    vv[:, :, 0], 0.1, out, kvg.decode_workspace(b.cache, b.seqs, 1))
        return [np.stack([b.keys_values(0, s)[j][b.ctxs[s]:] for s in range(B)]) for j in range(2)]

    a = fresh()
    k, v = a.rows(2), a.rows(2)
    k[0, 1, 0, 9], v[0, 1, 1, 9] = 300.0, 500.0                # sequence 0 or 1: large, and beyond the type's range
    want_k, want_v = stored(a, k, v)
    assert np.array_equal(want_v.reshape(v[0].shape), host(v[0].float().clamp(-448, 448).to(torch.float8_e4m3fn)))
    assert (want_v == 448).any() and np.isfinite(want_k).all()
    at, nan, inf = n * B - 1, float("nan"), float("inf")        # the last token
    v[0, at, 0, 3:7] = torch.tensor([inf, -inf, nan, 1e30], device="cuda", dtype=v.dtype)
    k[0, at, 1, 5] = nan
    got_k, got_v = (x.reshape(-1, 2, D) for x in stored(fresh(), k, v))
    want_k, want_v = (x.reshape(-1, 2, D) for x in (want_k, want_v))
    assert np.array_equal(got_v[at, 0, [3, 4, 6]], [448, -448, 448]) and np.isnan(got_v[at, 0, 5])
    want_v[at, 0, 3:7] = got_v[at, 0, 3:7]
    assert np.array_equal(got_v, want_v, equal_nan=True)
    pair = range(D) if call.endswith("normed") else (5, 5 + D // 2) if pairing == 0 else (4, 5)
    assert np.isnan(got_k[at, 1, list(pair)]).all()
    want_k[at, 1, list(pair)] = nan
    assert np.array_equal(got_k, want_k, equal_nan=True)


def test_relocated_fp8_keys_keep_nan(kvg):
    b = Batch([20], [0], (4, 2, 64), "fp8", seed=24, poison=3.0)
    append(b, kvg.rotary(), None, None, b.rows(2), b.rows(2), None)
    hdr = kvg.kvg_artifact_header_init(b.cache, 20, 0, kvg.rope())
    payload = torch.empty(hdr.payload_bytes, dtype=torch.uint8, device="cuda")

    def moved():
        kvg.kvg_deposit(b.cache, b.seqs.block_tables[0], 0, 20, payload)
        there = Batch([20], [0], (4, 2, 64), "fp8", seed=25, poison=3.0)
        kvg.kvg_graft(there.cache, hdr, payload, there.seqs.block_tables[0], 0, 77, kvg.KVG_GRAFT_ALLOW_RELOCATE)
        return there.keys_values(0, 0)[0]

    want = moved()
    b.cache.k_pool.view(torch.uint8)[0, int(b.table[0, 1]), 1, 2, 40] = 0x7F       # token 18
    want[18, 1, [8, 40]] = np.nan
    assert np.isfinite(want[:18]).all() and np.array_equal(moved(), want, equal_nan=True)


# ---------------------------------------------------------------------------- attention over one segment, few rows

@pytest.mark.parametrize("dtype,heads", [("bf16", (16, 8, 256)), ("bf16", (16, 2, 128)), ("bf16", (4, 4, 128)), ("bf16", (4, 2, 64)),
                                         ("fp8", (8, 4, 128)), ("fp8", (16, 8, 256))],
                         ids=lambda x: x if isinstance(x, str) else "x".join(map(str, x)))
@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("lens", ["tokens", "chunks"])
def test_few_rows_over_one_segment(kvg, dtype, heads, window, lens):
    """Batches that one segment holds, so that no launch is split: a small one takes four waves a workgroup (over up to four
    units of 128 keys; two waves at head_dim 64), one of many layers two.  Every row against the oracle, and the same bytes."""
    L, ctxs = 48, [0, 129, 256, 399, 480, 510, 127, 330]
    most = 32 * heads[1] // heads[0]                            # rows of 32 pairs
    n = [1] * 8 if lens == "tokens" else [1, most, 3, most - 1, 2, 1, most, 4]
    n = [min(x, most, 512 - c) for x, c in zip(n, ctxs)]
    one = Batch(n, ctxs, heads, dtype, layers=1, windows=(window,), seed=26)
    assert one.max_pages * 16 <= 512
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


# ---------------------------------------------------------------------------- attention over values that are not finite

@pytest.mark.parametrize("heads,lens,ctxs", [
    ((4, 2, 64), [200, 3], [10, 100]), ((8, 1, 128), [200, 3], [10, 100]), ((2, 1, 256), [200, 3], [10, 100]),    # tiles
    ((4, 2, 256), [300], [900]), ((8, 2, 128), [150, 1], [1500, 700]),                                            # split tiles
    ((16, 8, 256), [1, 2, 9, 1], [90, 70, 63, 400]), ((4, 4, 128), [32, 1], [60, 200]), ((8, 2, 64), [8, 1], [64, 71]),   # few rows
    ((16, 8, 256), [1, 4, 1], [1500, 700, 71])], ids=lambda x: "x".join(map(str, x)))
@pytest.mark.parametrize("window", [0, 60])
def test_fp8_nan_stays_with_the_rows_that_see_it(heads, lens, ctxs, window):
    """NaN codes (of both signs) among the values and keys of token 70 of every sequence that has it: rows that do not see it keep
    their bytes, rows that do are NaN, in that dimension (a value) or whole (a key)."""
    group = heads[0] // heads[1]
    for which, code in (("v", 0x7F), ("v", 0xFF), ("k", 0x7F), ("k", 0xFF)):
        b = Batch(lens, ctxs, heads, "fp8", windows=(window,) if window else None, seed=27)
        q = b.rows(heads[0], 2.0)
        want = b.attend(q, 0.1)
        assert want.float().isfinite().all()
        pool = (b.cache.v_pool if which == "v" else b.cache.k_pool).view(torch.uint8)
        for s, (n, c) in enumerate(zip(lens, ctxs)):
            if c + n > 70:
                pool[0, int(b.table[s, 70 // 16]), 0, 70 % 16, 5] = code
        got = b.attend(q, 0.1)
        for s, (n, c) in enumerate(zip(lens, ctxs)):
            for i in range(n):
                if c + i >= 70 and (not window or c + i < 70 + window):
                    hit = got[0, int(b.cu[s]) + i, :group]
                    assert (hit[:, 5] if which == "v" else hit).isnan().all(), (which, code, s, i)
                    hit[:, 5 if which == "v" else slice(None)] = want[0, int(b.cu[s]) + i, :group, 5 if which == "v" else slice(None)]
        assert torch.equal(bits(got), bits(want)), (which, code)


@pytest.mark.parametrize("dtype,heads,lens,ctxs", [
    ("bf16", (4, 2, 64), [100, 3], [0, 100]), ("bf16", (2, 1, 256), [130], [800]), ("bf16", (16, 8, 128), [1, 2], [90, 200]),
    ("f32", (4, 2, 64), [100, 1], [0, 300])], ids=lambda x: x if isinstance(x, str) else "x".join(map(str, x)))
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_keys_that_are_infinite(dtype, heads, lens, ctxs, sign):
    """A key with an infinite component scores Inf of one sign or the other: -Inf weighs 0, as if the key were not there; Inf leaves
    the row NaN."""
    b = Batch(lens, ctxs, heads, dtype, seed=28)
    q = b.rows(heads[0], 2.0)
    group, at = heads[0] // heads[1], 70
    want = b.attend(q, 0.1)
    for s in range(len(lens)):
        b.cache.k_pool[0, int(b.table[s, at // 16]), 0, at % 16, 5] = sign * math.inf
    got = b.attend(q, 0.1)
    seen = 0
    for s, (n, c) in enumerate(zip(lens, ctxs)):
        k, v = b.keys_values(0, s)
        without = np.arange(len(k)) != at
        k[at] = 0.0
        for i in range(n):
            t = int(b.cu[s]) + i
            if c + i < at:
                assert torch.equal(bits(got[0, t]), bits(want[0, t])), (s, i)
                continue
            assert torch.equal(bits(got[0, t, group:]), bits(want[0, t, group:])), (s, i)
            row = host(q[0, t:t + 1])[:, :group]
            exact, tol = attention_bound(row, np.array([c + i - 1]), k[without, :1], v[without, :1], 0.1, 0, dtype)
            for h in range(group):
                if float(q[0, t, h, 5]) * sign > 0:
                    assert got[0, t, h].isnan().all(), (s, i, h)
                else:
                    seen += 1
                    assert np.all(np.abs(host(got[0, t, h]) - exact[0, h]) <= tol[0, h]), (s, i, h)
    assert seen > 0
