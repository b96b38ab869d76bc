"""Rotary positions with several axes on the GPU, alone and with the norms and the append, against the oracle in fp64."""

import numpy as np
import pytest
import torch

from oracle import packed as oracle
from tests.packed_helpers import TORCH, U, Batch, host
from tests.test_gpu_packed import PAIRINGS, SCALED, SCALINGS, bits, kvg, pair_size, rotated_bound  # noqa: F401

pytestmark = pytest.mark.gpu


def plan(kvg, pairs, order, own, pairing, dim, scaling, pos, amplitude=1.25):  # noqa: F811
    rt = kvg.rotary(10000.0, PAIRINGS.index(pairing), dim, SCALINGS.index(scaling), amplitude=amplitude, **SCALED)
    axes = kvg.Axes(pos, pairs, {"sections": kvg.KVG_AXES_SECTIONS, "turns": kvg.KVG_AXES_TURNS}[order], own)
    theta = oracle.axes_frequencies(pairs, 10000.0, own, scaling=scaling, **SCALED)
    return rt, axes, theta, oracle.axis_of_pairs(pairs, order)


PLANS = [((8, 12, 12), "sections", False, "half", 0, "plain"), ((12, 10, 10), "turns", False, "half", 0, "rotations"),
         ((8, 12, 12), "sections", True, "interleaved", 0, "linear"), ((5, 7, 1, 3), "turns", False, "interleaved", 32, "index"),
         ((15, 1), "sections", True, "half", 32, "rotations"), ((32,), "sections", True, "half", 0, "base"),
         ((2, 6), "sections", True, "interleaved", 16, "base")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,order,own,pairing,dim,scaling", PLANS)
@pytest.mark.parametrize("head_dim,tokens,heads", [(64, 1, 1), (64, 83, 5), (256, 19, 24)])
def test_rotate_axes(kvg, dtype, pairs, order, own, pairing, dim, scaling, head_dim, tokens, heads):  # noqa: F811
    scale = 1 if dim else head_dim // 64
    pairs = tuple(p * scale for p in pairs)
    gen = torch.Generator(device="cuda").manual_seed(7)
    pos = torch.randint(-50, 3_000_000, (len(pairs), tokens), generator=gen, device="cuda")
    rt, axes, theta, axis = plan(kvg, pairs, order, own, pairing, dim, scaling, pos)
    wide = torch.randn(tokens, heads + 3, head_dim, generator=gen, device="cuda").to(TORCH[dtype])
    x = wide[:, 1:1 + heads]
    y = torch.full((tokens, heads, head_dim), 7.0, dtype=TORCH[dtype], device="cuda")
    kvg.kvg_rotate_axes(rt, axes, x, y)
    want = oracle.rotate_axes(host(x), pos.cpu().numpy(), theta, axis, pairing, 1.25)
    size = 1.25 * pair_size(host(x), 2 * len(theta), pairing)
    assert np.all(np.abs(host(y) - want) <= rotated_bound(want, size, dtype))
    assert torch.equal(y[..., 2 * len(theta):], x[..., 2 * len(theta):])          # left as they are
    kvg.kvg_rotate_axes(rt, axes, x, x)                                            # in place, strided
    assert torch.equal(x, y)


def test_one_position_on_every_axis_is_the_plain_rotary(kvg):  # noqa: F811
    x = torch.randn(40, 6, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(40, device="cuda") * 977
    y, z = torch.empty_like(x), torch.empty_like(x)
    rt = kvg.rotary(scaling=kvg.KVG_ROTARY_ROTATIONS, **SCALED)
    kvg.kvg_rotate(rt, pos, x, y)
    for order in (kvg.KVG_AXES_SECTIONS, kvg.KVG_AXES_TURNS):
        kvg.kvg_rotate_axes(rt, kvg.Axes(pos.repeat(3, 1), (24, 20, 20), order), x, z)
        assert torch.equal(bits(y), bits(z))


def test_gradient_is_the_rotation_at_negated_positions(kvg):  # noqa: F811
    """<R x, g> = <x, R' g> for all g, so R' g is the gradient; against differences of a loss in fp64 as well."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    pos = torch.randint(0, 5000, (3, 9), generator=gen, device="cuda")
    rt, axes, theta, axis = plan(kvg, (8, 12, 12), "sections", False, "half", 0, "plain", pos, amplitude=1.0)
    x, g = (torch.randn(9, 2, 64, generator=gen, device="cuda") for _ in range(2))
    grad = torch.empty_like(g)
    kvg.kvg_rotate_axes(rt, kvg.Axes(-pos, (8, 12, 12)), g, grad)
    p, gh = pos.cpu().numpy(), host(g)
    want = oracle.rotate_axes(gh, -p, theta, axis, "half")
    size = pair_size(gh, 64, "half")
    assert np.all(np.abs(host(grad) - want) <= rotated_bound(want, size, "f32"))
    loss = lambda a: float((oracle.rotate_axes(a, p, theta, axis, "half") * gh).sum())  # noqa: E731
    xh = host(x)
    for t, h, d in ((0, 0, 0), (4, 1, 37), (8, 0, 63)):
        e = np.zeros_like(xh)
        e[t, h, d] = 0.5                                       # the loss is linear: any step gives the gradient
        slope = loss(xh + e) - loss(xh - e)
        assert abs(slope - float(grad[t, h, d])) <= float(rotated_bound(want, size, "f32")[t, h, d]) + 1e-10


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("heads,pairs,order,own,pairing,dim,wide", [
    ((4, 2, 64), (8, 12, 12), "sections", False, "half", 0, 0), ((8, 8, 128), (12, 10, 10), "turns", False, "interleaved", 64, 6),
    ((16, 2, 256), (32, 48, 48), "sections", True, "half", 0, 4)])
def test_norm_append_axes(kvg, dtype, heads, pairs, order, own, pairing, dim, wide):  # noqa: F811
    Hq, Hkv, D = heads
    b = Batch([3, 0, 1, 40, 17], [0, 5, 31, 16, 250], heads, dtype, layers=2, seed=5, lead=2, tail=3, poison=3.0)
    pos = torch.randint(0, 200_000, (len(pairs), b.tokens), generator=b.gen, device="cuda")
    rt, axes, theta, axis = plan(kvg, pairs, order, own, pairing, dim, "plain", pos, 1.1)
    q, k, v = b.rows(Hq, 1.5, wide), b.rows(Hkv, 1.5, wide), b.rows(Hkv, 1.5, wide)
    qw, kw = (torch.randn(2, D, generator=b.gen, device="cuda").mul(0.2).to(TORCH[b.raw]) for _ in range(2))
    before = b.cache.k_pool.clone(), b.cache.v_pool.clone()
    out = torch.full((2, b.tokens, Hq, D), 7.0, dtype=TORCH[b.raw], device="cuda")
    kvg.kvg_norm_append_axes(b.cache, b.seqs, b.packed, rt, axes, kvg.HeadNorm(qw, kw, 1e-6, 1.0), 0, 2, q, k, v, out)
    p = pos.cpu().numpy()
    seen = torch.zeros(before[0].shape[1], 16, dtype=torch.bool)
    rel = (D + 12) * U                                         # of a norm: the sum of squares, its root, two products
    for l in range(2):
        for i, n in enumerate(b.lens):
            r0 = int(b.cu[i])
            rows = slice(r0, r0 + n)
            for raw, w, got in ((q, qw, None), (k, kw, b.cache.k_pool)):
                x = oracle.rms_norm(host(raw[l, rows]), host(w[l]), 1e-6, 1.0)
                want = oracle.rotate_axes(x, p[:, rows], theta, axis, pairing, 1.1)
                size = pair_size(x, 2 * len(theta), pairing) * 1.1
                if got is None:
                    assert np.all(np.abs(host(out[l, rows]) - want) <= rotated_bound(want, size, b.raw, rel))
                    continue
                for t in range(n):
                    at = b.ctxs[i] + t
                    page = int(b.table[i, at // 16])
                    seen[page, at % 16] = True
                    have = host(got[l, page, :, at % 16])
                    assert np.all(np.abs(have - want[t]) <= rotated_bound(want[t], size[t], dtype, rel))
                    stored = v[l, r0 + t].float().to(TORCH[dtype])
                    assert torch.equal(bits(b.cache.v_pool[l, page, :, at % 16]), bits(stored))
    for pool, was in zip((b.cache.k_pool, b.cache.v_pool), before):      # the other rows keep their bytes
        keep = ~seen.cuda()[None, :, None, :, None]
        assert bool(((bits(pool) == bits(was)) | ~keep).all())
    outside = torch.from_numpy(b.outside()).cuda()
    assert bool((out[:, outside] == 7.0).all())
    # one position on every axis: kvg_norm_append's bytes
    if not own:
        again = torch.full_like(out, 7.0)
        start = b.start.copy()
        flat = np.zeros((len(pairs), b.tokens), dtype=np.int64)
        for i, n in enumerate(b.lens):
            flat[:, b.cu[i]:b.cu[i] + n] = start[i] + b.ctxs[i] + np.arange(n)
        same = kvg.Axes(torch.from_numpy(flat).cuda(), axes.pairs, axes.order, False)
        norm = kvg.HeadNorm(qw, kw, 1e-6, 1.0)
        kvg.kvg_norm_append_axes(b.cache, b.seqs, b.packed, rt, same, norm, 0, 2, q, k, v, out)
        pools = b.cache.k_pool.clone(), b.cache.v_pool.clone()
        kvg.kvg_norm_append(b.cache, b.seqs, b.packed, rt, norm, 0, 2, q, k, v, again)
        assert torch.equal(bits(out), bits(again))
        assert torch.equal(bits(pools[0]), bits(b.cache.k_pool)) and torch.equal(bits(pools[1]), bits(b.cache.v_pool))
