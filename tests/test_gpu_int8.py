"""8-bit integer caches on the GPU: append and attention against the oracle in fp64, at the lengths, masks, strides, scales
and metadata where they can go wrong."""

import math

import numpy as np
import pytest
import torch

from oracle import int8 as oracle
from oracle import packed as oracle_packed
from tests.int8_helpers import Int8Batch, check
from tests.packed_helpers import U, host
from tests.test_gpu_axes import plan
from tests.test_gpu_packed import bits, kvg, make_rotary, pair_size, rotated_bound  # noqa: F401

pytestmark = pytest.mark.gpu

LENS = [5, 1, 0, 40, 17, 1]
CTXS = [0, 0, 9, 16, 250, 1200]


# ---------------------------------------------------------------------------- attention

@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 2, 128), (8, 2, 128), (16, 2, 64), (16, 8, 256), (8, 1, 256)])
@pytest.mark.parametrize("lens,ctxs", [([1], [0]), ([1], [15]), ([1, 1, 1], [16, 511, 700]), ([17], [0]), ([33, 2], [31, 512]), (LENS, CTXS)])
def test_attention(kvg, heads, lens, ctxs):  # noqa: F811
    b = Int8Batch(lens, ctxs, heads, seed=11, lead=1, tail=2)
    q = b.rows(heads[0], 2.0)
    check(b, q, b.attend(q, 1.0 / math.sqrt(heads[2])), 1.0 / math.sqrt(heads[2]))


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 4, 128), (8, 4, 256)])
@pytest.mark.parametrize("window", [1, 16, 100, 513])
def test_windows(kvg, heads, window):  # noqa: F811
    b = Int8Batch(LENS, CTXS, heads, layers=3, windows=(window, 0, window), seed=5)
    q = b.rows(heads[0], 2.0, wide=4)
    check(b, q, b.attend(q, 1.0 / math.sqrt(heads[2])), 1.0 / math.sqrt(heads[2]))


@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128), (16, 8, 256)])
def test_long_prompts(kvg, heads):  # noqa: F811
    """Whole walks in one workgroup (many tiles), and splits over segments."""
    for lens, ctxs in (([1500, 1300, 700, 900, 3, 1], [0, 100, 0, 7, 3000, 4000]), ([200], [4500]), ([1], [9000])):
        b = Int8Batch(lens, ctxs, heads, seed=2)
        q = b.rows(heads[0], 2.0)
        rows = lambda n: (0, 1, 63, 64, n // 2, n - 2, n - 1)  # noqa: E731
        check(b, q, b.attend(q, 1.0 / math.sqrt(heads[2])), 1.0 / math.sqrt(heads[2]), rows)


@pytest.mark.parametrize("heads,far", [((4, 2, 64), False), ((16, 8, 256), False), ((4, 2, 128), False), ((4, 2, 128), True), ((8, 4, 256), True)])
def test_a_rows_bytes_are_its_own(kvg, heads, far):  # noqa: F811
    """The same cache read in one call, in chunks, token by token and alone: the same bytes.  Scales differ a thousandfold; `far`: every
    other row's scores are past 2^20, and value scales far from 1."""
    n = 700
    b = Int8Batch([n, 30], [0, 1100], heads, seed=4, spread=3.0)
    q, scale = b.rows(heads[0], 2.0), 0.1
    if far:
        q[:, ::2] *= 2.0 ** 22
        b.cache.v_scale.mul_(2.0 ** 20)
        assert bool(b.attend(q, scale)[:, :n].isfinite().all())
    whole = b.attend(q, scale)
    for cuts in ([1, 64, 65, 300, 270], [n - 1, 1], [35] * 20):
        at = 0
        for c in cuts:
            seqs = kvg.Seqs(b.seqs.block_tables[:1].contiguous(), torch.tensor([at], dtype=torch.int32, device="cuda"), b.seqs.start_pos[:1], at)
            packed = kvg.Packed(torch.tensor([0, c], dtype=torch.int32, device="cuda"), c, c)
            part = q[:, at:at + c].contiguous()
            out = torch.empty_like(part)
            kvg.kvg_int8_attn(b.cache, seqs, packed, 0, 1, part, scale, out, kvg.int8_attn_workspace(b.cache, seqs, packed, 1))
            assert torch.equal(bits(out), bits(whole[:, at:at + c])), (cuts, at)
            at += c
    for at in (0, 1, 15, 16, 511, 512, 699):                   # single tokens beside others
        seqs = kvg.Seqs(b.seqs.block_tables, torch.tensor([at, 1100], dtype=torch.int32, device="cuda"), b.seqs.start_pos, 1100)
        packed = kvg.Packed(torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 2, 1)
        part = torch.cat([q[:, at:at + 1], q[:, n:n + 1]], dim=1)
        out = torch.empty_like(part)
        kvg.kvg_int8_attn(b.cache, seqs, packed, 0, 1, part, scale, out, kvg.int8_attn_workspace(b.cache, seqs, packed, 1))
        assert torch.equal(bits(out[:, 0]), bits(whole[:, at])) and torch.equal(bits(out[:, 1]), bits(whole[:, n]))


def test_scales_far_apart(kvg):  # noqa: F811
    """Value scales from 2^-60 to 2^60, key scales that leave one page heavy, and blocks of zeros."""
    for heads, lens, ctxs in (((4, 2, 64), [60, 1, 1], [0, 100, 700]), ((8, 4, 256), [40, 1], [30, 600]), ((4, 4, 128), [300], [500])):
        b = Int8Batch(lens, ctxs, heads, seed=9)
        rng = np.random.default_rng(3)
        b.cache.v_scale.copy_(torch.from_numpy(2.0 ** rng.integers(-60, 61, b.cache.v_scale.shape)).float())
        zero = torch.from_numpy(rng.random(b.cache.v_scale.shape) < 0.2).cuda()
        b.cache.v_scale[zero] = 0.0
        b.cache.k_scale[torch.from_numpy(rng.random(b.cache.v_scale.shape) < 0.2).cuda()] = 0.0
        q = b.rows(heads[0], 2.0)
        check(b, q, b.attend(q, 0.1), 0.1)
        b.cache.v_scale.zero_()
        assert bool((b.attend(q, 0.1) == 0).all())


def test_extreme_queries(kvg):  # noqa: F811
    b = Int8Batch([20, 1], [5, 600], (4, 2, 128), seed=1)
    q = b.rows(4, 1.0)
    q[0, 3] = 0.0                                              # equal weights
    q[0, 4, :, 1:] = 0.0                                       # one component
    q[0, 5] *= 2.0 ** -60
    q[0, 6, :, 0] = 300.0                                      # one far larger than the others
    q[0, 7, 0] = 1e-39
    check(b, q, b.attend(q, 0.09), 0.09)
    want = b.attend(q, 0.09)
    bad = q.clone()
    bad[0, 2, 1, 7], bad[0, 8, 3, 100], bad[0, 20, 0, 0] = float("nan"), float("inf"), -float("inf")
    out = b.attend(bad, 0.09)
    for t, h in ((2, 1), (8, 3), (20, 0)):
        assert bool(out[0, t, h].isnan().all())
        want[0, t, h] = out[0, t, h]
    assert torch.equal(bits(out), bits(want))


@pytest.mark.parametrize("heads,lens,ctxs", [((4, 2, 64), [50], [0]), ((8, 4, 256), [3], [30]), ((4, 4, 128), [200], [600])])
def test_scores_past_fp32(kvg, heads, lens, ctxs):  # noqa: F811
    """Scores that leave fp32: the key with the largest takes the row, or the keys where they are equal."""
    b = Int8Batch(lens, ctxs, heads, seed=12)
    b.cache.k_scale[0, int(b.table[0, 0])] = 1e35
    b.cache.k_scale[0, int(b.table[0, 1])] = 0.0
    q = b.rows(heads[0], 1e25)
    out = host(b.attend(q, 0.1)[0])
    kn, ks, vn, vs = b.cached(0, 0)
    group = heads[0] // heads[1]
    for t in range(lens[0]):
        n = ctxs[0] + t + 1
        for h in range(heads[0]):
            g = h // group
            s = kn[:n, g] @ host(q[0, t, h]) * ks[:n, g]
            top = s >= s.max() - 1e-9 * abs(s.max())
            want = (vn[:n, g] * vs[:n, g, None])[top].mean(axis=0)
            assert np.all(np.abs(out[t, h] - want) <= 2.0 ** -7 * np.abs(vn[:n, g] * vs[:n, g, None])[top].max(axis=0) + 1e-30), (t, h)


@pytest.mark.parametrize("heads,lens,ctxs", [((4, 2, 64), [50, 1], [0, 300]), ((8, 4, 256), [200], [0]), ((4, 4, 128), [5, 7], [700, 0])])
@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
def test_scales_that_are_not_finite(kvg, heads, lens, ctxs, which):  # noqa: F811
    """Rows that see a token of such a page are NaN, the others keep their bytes."""
    b = Int8Batch(lens, ctxs, heads, seed=8)
    q = b.rows(heads[0], 2.0)
    want = b.attend(q, 0.1)
    for value in (float("nan"), float("inf")):
        page = int(b.table[0, 1])
        old = getattr(b.cache, which)[0, page, 1].clone()
        getattr(b.cache, which)[0, page, 1] = value
        out = b.attend(q, 0.1)
        group = heads[0] // heads[1]
        for t in range(lens[0]):
            if ctxs[0] + t >= 16:
                assert bool(out[0, t, group:2 * group].isnan().all())
                want[0, t, group:2 * group] = out[0, t, group:2 * group]
        assert torch.equal(bits(out), bits(want))
        getattr(b.cache, which)[0, page, 1] = old
        want = b.attend(q, 0.1)


def test_bad_metadata_is_skipped(kvg):  # noqa: F811
    b = Int8Batch([8, 4, 6], [20, 0, 33], (4, 2, 64), seed=6, tail=3)
    q = b.rows(4, 2.0)
    want = b.attend(q, 0.1)
    for edit in ("ctx", "cu", "pages"):
        c = Int8Batch([8, 4, 6], [20, 0, 33], (4, 2, 64), seed=6, tail=3)
        if edit == "ctx":
            c.seqs.ctx_lens[1] = -5
        elif edit == "cu":
            c.packed.cu_tokens[2] = 5                          # descends, and the next holds more than max_len
        else:
            c.seqs.block_tables[1, 0] = 1 << 30
        out = c.attend(q, 0.1)
        assert torch.equal(bits(out[:, :8]), bits(want[:, :8]))
        assert bool((out[:, 18:] == 7.0).all())


# ---------------------------------------------------------------------------- append

def run_append(b, rt, norm, q, k, v, out, axes=None):
    b.kvg.kvg_int8_append(b.cache, b.seqs, b.packed, rt, norm, 0, b.layers, q, k, v, out, axes=axes)


def fp32_integers(x, scale):
    """The kernel's rounding of fp32 values, in fp32."""
    inv = np.float32(1.0) / scale
    return np.clip(np.rint(x * inv), -127, 127)


@pytest.mark.parametrize("heads,pairing,dim,scaling,wide,axes", [
    ((4, 2, 64), "half", 0, "plain", 0, False), ((8, 8, 128), "interleaved", 64, "index", 6, False), ((16, 2, 256), "half", 128, "rotations", 4, False),
    ((2, 1, 256), "interleaved", 0, "linear", 0, True), ((4, 4, 128), "half", 0, "plain", 2, True)])
@pytest.mark.parametrize("normed", [True, False])
def test_append(kvg, heads, pairing, dim, scaling, wide, axes, normed):  # noqa: F811
    Hq, Hkv, D = heads
    lens, ctxs = [3, 0, 1, 40, 17, 1], [0, 5, 31, 16, 250, 7]
    b = Int8Batch(lens, ctxs, heads, layers=2, seed=5, lead=2, tail=3, poison=1.0)
    theta, pos = None, None
    if axes:
        pos = torch.randint(0, 9000, (3, b.tokens), generator=b.gen, device="cuda")
        pairs = tuple(D // 2 * x // 32 for x in (8, 12, 12))
        rt, ax, theta, axis = plan(kvg, pairs, "sections", pairing == "interleaved", pairing, dim, scaling, pos, 1.1)
    else:
        rt, theta = make_rotary(kvg, D, pairing, dim, scaling, amplitude=1.1)
        ax = None
    q, k, v = b.rows(Hq, 1.5, wide), b.rows(Hkv, 1.5, wide), b.rows(Hkv, 1.5, wide)
    k[:, 5:9] *= 0.05                                          # some pages grow a lot, some not at all
    v[:, 2] *= 8.0
    qw, kw = (torch.randn(2, D, generator=b.gen, device="cuda").mul(0.2).to(torch.bfloat16) for _ in range(2))
    norm = kvg.HeadNorm(qw, kw, 1e-6, 1.0) if normed else None
    before = [t.clone() for t in b.cache.tensors()]
    out = torch.full((2, b.tokens, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    run_append(b, rt, norm, q, k, v, out, ax)
    rel = (D + 12) * U if normed else 0.0
    kp, vp, ksc, vsc = (t.cpu().numpy() for t in b.cache.tensors())
    kp0, vp0, ksc0, vsc0 = (t.cpu().numpy() for t in before)
    touched = {}
    for l in range(2):
        for i, n in enumerate(lens):
            rows = slice(int(b.cu[i]), int(b.cu[i]) + n)
            if n == 0:
                continue
            p = pos[:, rows].cpu().numpy() if axes else b.start[i] + ctxs[i] + np.arange(n)
            turned = []
            for raw, w in ((q, qw), (k, kw)):
                x = host(raw[l, rows])
                x = oracle_packed.rms_norm(x, host(w[l]), 1e-6, 1.0) if normed else x
                y = oracle_packed.rotate_axes(x, p, theta, axis, pairing, 1.1) if axes else oracle_packed.rotate(x, p, theta, pairing, 1.1)
                turned.append((y, pair_size(x, 2 * len(theta), pairing) * 1.1))
            want, size = turned[0]
            assert np.all(np.abs(host(out[l, rows]) - want) <= rotated_bound(want, size, "bf16", rel))
            for first in range(ctxs[i] - ctxs[i] % 16, ctxs[i] + n, 16):
                t0, t1 = max(first, ctxs[i]), min(first + 16, ctxs[i] + n)
                page, held, new = int(b.table[i, first // 16]), t0 - first, slice(t0 - ctxs[i], t1 - ctxs[i])
                touched.setdefault(page, (held, held + t1 - t0))
                for h in range(Hkv):
                    # keys: within the error of the fp32 norm and rotation, u of the largest
                    y, size = turned[1][0][new, h], turned[1][1][new, h]
                    off = (4 * U + 1.5 * rel) * size.max() + U * np.abs(y).max()
                    _, _, s = oracle.append_page(kp0[l, page, h, :held].astype(float), float(ksc0[l, page, h]), y)
                    got = float(ksc[l, page, h])
                    assert abs(got - s) <= off / 127 + 2 * U * s
                    assert np.all(np.abs(kp[l, page, h, held:held + t1 - t0] * got - y) <= got * (0.5 + 127 * 4 * U) + off)
                    # values: the same operations in fp32
                    x = v[l, rows][new, h].float().cpu().numpy()
                    s = np.float32(np.abs(x).max()) / np.float32(127)
                    s = max(s, vsc0[l, page, h]) if held else s
                    assert vsc[l, page, h] == s
                    assert np.array_equal(vp[l, page, h, held:held + t1 - t0], fp32_integers(x, s))
                    for pool, pool0, sc, sc0 in ((kp, kp0, ksc, ksc0), (vp, vp0, vsc, vsc0)):
                        r = sc0[l, page, h] / sc[l, page, h]
                        was = pool0[l, page, h, :held].astype(np.float32)
                        assert np.array_equal(pool[l, page, h, :held], np.rint(was * r) if held and r != 1 else was)
    for pool, pool0, sc, sc0 in ((kp, kp0, ksc, ksc0), (vp, vp0, vsc, vsc0)):      # everything else keeps its bytes
        for page in range(pool.shape[1]):
            end = touched[page][1] if page in touched else 0
            assert np.array_equal(pool[:, page, :, end:], pool0[:, page, :, end:])
            if page not in touched:
                assert np.array_equal(sc[:, page], sc0[:, page])
    assert bool((out[:, torch.from_numpy(b.outside()).cuda()] == 7.0).all())


def test_append_token_by_token(kvg):  # noqa: F811
    """A page filled a token at a time: every value within half a step for each time its page's scale grew, plus one."""
    b = Int8Batch([1], [0], (2, 2, 64), seed=3, max_pages=3)
    rows = torch.randn(1, 40, 2, 64, generator=b.gen, device="cuda")
    rows *= torch.linspace(0.2, 3.0, 40, device="cuda")[None, :, None, None]
    v = rows.to(torch.bfloat16)
    grew = np.zeros((40, 2))
    last = None
    for t in range(40):
        b.seqs.ctx_lens[0] = t
        seqs = kvg.Seqs(b.seqs.block_tables, b.seqs.ctx_lens, b.seqs.start_pos, t)
        one = v[:, t:t + 1].contiguous()
        kvg.kvg_int8_append(b.cache, seqs, b.packed, kvg.rotary(), None, 0, 1, None, one, one, None)
        scale = b.cache.v_scale[0, b.table[0, t // 16]].cpu().numpy()
        if t % 16:
            grew[t - t % 16:t] += scale > last
        last = scale
    b.ctxs, b.lens = [40], [0]
    _, _, n, s = b.cached(0, 0)
    err = np.abs(n * s[..., None] - host(v[0])).max(axis=2)
    assert np.all(err <= s * (grew + 1) * 0.5 * (1 + 1e-5))
    assert np.abs(n[32:40]).max() == 127


def test_append_edges(kvg):  # noqa: F811
    """Zeros, the smallest and largest values, Inf and NaN; keys and values alone; a page that comes to a sequence again."""
    b = Int8Batch([16], [0], (2, 2, 64), seed=3)
    page = int(b.table[0, 0])
    rt = kvg.rotary()
    k = torch.zeros(1, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    v[0, 3, 1, 5] = 2.0 ** -130                                # a scale below 2^-126 is raised to it
    run_append(b, rt, None, None, k, v, None)
    assert bool((b.cache.k_pool[0, page] == 0).all()) and bool((b.cache.k_scale[0, page] == 0).all())
    assert float(b.cache.v_scale[0, page, 0]) == 0.0 and float(b.cache.v_scale[0, page, 1]) == 2.0 ** -126
    v.normal_(generator=b.gen)
    v[0, 3, 1, 5] = 3.0e38
    run_append(b, rt, None, None, k, v, None)
    assert int(b.cache.v_pool[0, page, 1, 3, 5]) == 127 and math.isfinite(float(b.cache.v_scale[0, page, 1]))
    for bad in (float("nan"), float("inf"), -float("inf")):
        w = v.clone()
        w[0, 9, 0, 1] = bad
        run_append(b, rt, None, None, k, w, None)
        assert math.isnan(float(b.cache.v_scale[0, page, 0])) and math.isfinite(float(b.cache.v_scale[0, page, 1]))
    # tokens 4 .. 15 again: the page has held rows, so it stays NaN; the whole page again: it is new
    part = kvg.Packed(torch.tensor([0, 12], dtype=torch.int32, device="cuda"), 12, 12)
    seqs = kvg.Seqs(b.seqs.block_tables, torch.tensor([4], dtype=torch.int32, device="cuda"), b.seqs.start_pos, 4)
    kvg.kvg_int8_append(b.cache, seqs, part, rt, None, 0, 1, None, k[:, 4:].contiguous(), v[:, 4:].contiguous(), None)
    assert math.isnan(float(b.cache.v_scale[0, page, 0]))
    run_append(b, rt, None, None, k, v, None)
    assert math.isfinite(float(b.cache.v_scale[0, page, 0]))


def test_append_then_attend_is_close_to_bf16(kvg):  # noqa: F811
    """The same prompt through a bf16 and an int8 cache: outputs apart by the cache's rounding (0.8% of a Gaussian row) alone."""
    heads = (8, 4, 128)
    b = Int8Batch([300, 45], [0, 0], heads, seed=7)
    q, k, v = b.rows(8), b.rows(4), b.rows(4)
    rt = kvg.rotary()
    out = torch.empty_like(q)
    run_append(b, rt, None, q, k, v, out)
    got = b.attend(out, 0.09)
    cache = kvg.Cache.allocate(1, b.cache.n_pages, 8, 4, 128, torch.bfloat16)
    other = torch.empty_like(q)
    kvg.kvg_norm_append(cache, b.seqs, b.packed, rt, None, 0, 1, q, k, v, other)
    assert torch.equal(bits(out), bits(other))
    want = torch.empty_like(q)
    kvg.kvg_packed_attn(cache, b.seqs, b.packed, 0, 1, other, 0.09, want, kvg.packed_attn_workspace(cache, b.seqs, b.packed, 1))
    rel = float((got.float() - want.float()).norm() / want.float().norm())
    assert rel < 0.03, rel
