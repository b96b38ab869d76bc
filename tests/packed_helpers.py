"""Batches of packed sequences for the GPU tests, their numpy copies, and the error bounds (test infrastructure)."""

import numpy as np
import torch

from oracle import packed as oracle

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24, "fp8": 2.0 ** -4}     # of a rounding, relative to the value
U = 2.0 ** -24


def host(t):
    """A tensor's values in fp64 (numpy)."""
    return t.detach().cpu().to(torch.float64).numpy() if t.dtype != torch.float8_e4m3fn else t.detach().cpu().float().double().numpy()


class Batch:
    """Sequences with `lens` new tokens over `ctxs` cached ones, in a cache of pages in random order whose other pages,
    and rows past the tokens, hold `poison` (default NaN)."""

    def __init__(self, lens, ctxs, heads=(4, 2, 64), dtype="bf16", layers=1, windows=None, seed=0, lead=0, tail=0,
                 poison=float("nan"), k_sigma=1.0, spare_pages=3):
        from paper_2607_14431_amd import kvg
        self.kvg, self.dtype, self.heads, self.layers, self.windows = kvg, dtype, heads, layers, windows
        self.lens, self.ctxs = list(lens), list(ctxs)
        Hq, Hkv, D = heads
        rng = np.random.default_rng(seed)
        self.rng = rng
        B = len(lens)
        self.max_pages = max(-(-max(c + n, 1) // 16) for c, n in zip(ctxs, lens))
        n_pages = B * self.max_pages + spare_pages
        self.table = rng.permutation(n_pages)[:B * self.max_pages].reshape(B, self.max_pages).astype(np.int32)
        self.raw = "f32" if dtype == "f32" else "bf16"
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.gen = gen
        pools = []
        for j in range(2):
            x = torch.empty((layers, n_pages, Hkv, 16, D), dtype=torch.float32, device="cuda")
            x.normal_(0.0, k_sigma if j == 0 else 1.0, generator=gen)
            known = torch.zeros((n_pages, 16), dtype=torch.bool)
            for b in range(B):
                for t in range(self.ctxs[b] + self.lens[b]):
                    known[self.table[b, t // 16], t % 16] = True
            x.masked_fill_(~known.cuda()[None, :, None, :, None], poison)
            pools.append(x.to(TORCH[dtype]))
        self.cache = kvg.Cache(pools[0], pools[1], Hq, windows)
        self.cu = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int32) + lead
        self.tokens = int(self.cu[-1]) + tail
        self.start = rng.integers(0, 5000, B).astype(np.int64)
        self.seqs = kvg.Seqs(torch.from_numpy(self.table).cuda(), torch.tensor(self.ctxs, dtype=torch.int32, device="cuda"),
                             torch.from_numpy(self.start).cuda(), max(self.ctxs))
        self.packed = kvg.Packed(torch.from_numpy(self.cu).cuda(), self.tokens, max(self.lens))

    def rows(self, heads, sigma=1.0, wide=0, layers=None):
        """Random rows [layers][tokens][heads][D] of the raw dtype; wide > 0: a view into rows `wide` heads wider."""
        D = self.heads[2]
        x = torch.empty((layers or self.layers, self.tokens, heads + wide, D), dtype=torch.float32, device="cuda")
        x = x.normal_(0.0, sigma, generator=self.gen).to(TORCH[self.raw])
        return x[:, :, wide // 2:wide // 2 + heads] if wide else x

    def workspace(self):
        return self.kvg.packed_attn_workspace(self.cache, self.seqs, self.packed, self.layers)

    def attend(self, q, scale, out=None, ws=None):
        if out is None:
            out = torch.full((self.layers, self.tokens, self.heads[0], self.heads[2]), 7.0, dtype=TORCH[self.raw], device="cuda")
        self.kvg.kvg_packed_attn(self.cache, self.seqs, self.packed, 0, self.layers, q, scale, out,
                                 self.workspace() if ws is None else ws)
        return out

    def keys_values(self, l, b):
        """Sequence b's cached keys and values in layer l, [S][Hkv][D] fp64."""
        n = self.ctxs[b] + self.lens[b]
        pages = torch.from_numpy(self.table[b, :-(-n // 16)].astype(np.int64)).cuda()
        res = []
        for pool in (self.cache.k_pool, self.cache.v_pool):
            x = pool[l].view(torch.uint8)[pages].view(pool.dtype) if pool.dtype == torch.float8_e4m3fn else pool[l][pages]
            res.append(host(x).transpose(0, 2, 1, 3).reshape(-1, *self.heads[1:])[:n])
        return res

    def outside(self):
        """Packed rows that belong to no sequence."""
        mine = np.zeros(self.tokens, dtype=bool)
        for b, n in enumerate(self.lens):
            mine[self.cu[b]:self.cu[b] + n] = True
        return np.flatnonzero(~mine)


def attention_bound(q, index, k, v, scale, window, dtype):
    """(want, tol) of attention rows, per element.  With D products a score is off by at most (D + 4) u of the sum of their
    sizes (u = 2^-24: every product and sum rounds once, the scale and its product with log2 e twice more), and a
    weight's exponential by 4 u more (2 of the argument near 0, 2 of exp2).  Weights round to bf16 on the bf16 matrix
    cores, at most half a step h = 2^-8 each, and are normalised by the sum of the rounded weights: out' - out =
    sum w_j d_j (v_j - out) / (1 + sum w_j d_j), |d_j| <= h + the above.  The sums of n terms add n u of the
    sizes summed; the result rounds once to the raw type."""
    want, spread, mass, score = oracle.attend_bounds(q, index, k, v, scale, window)
    D, n = q.shape[2], k.shape[0]
    h = 2.0 ** -8 if dtype != "f32" else 0.0
    off = ((h + 8 * U) * spread + (D + 4) * U * score) * 1.02 + (n + 8) * U * (mass + np.abs(want))
    return want, off + HALF_STEP["f32" if dtype == "f32" else "bf16"] * (np.abs(want) + off) + 1e-37


def check_attention(batch, q, out, scale, rows_of=lambda n: range(n), l_list=None):
    """Every sequence's rows against the oracle; rows of no sequence keep the fill value 7."""
    worst = 0.0
    for l in l_list if l_list is not None else range(batch.layers):
        w = batch.windows[l] if batch.windows else 0
        for b, n in enumerate(batch.lens):
            idx = np.array(sorted(set(i for i in rows_of(n) if 0 <= i < n)), dtype=np.int64)
            if len(idx) == 0:
                continue
            k, v = batch.keys_values(l, b)
            r = torch.from_numpy(idx + int(batch.cu[b])).cuda()
            want, tol = attention_bound(host(q[l][r]), idx + batch.ctxs[b], k, v, scale, w, batch.dtype)
            got = host(out[l][r])
            assert np.isfinite(got).all(), f"layer {l} sequence {b}: not finite"
            ratio = np.abs(got - want) / tol
            worst = max(worst, float(ratio.max()))
            at = np.unravel_index(int(ratio.argmax()), ratio.shape)
            assert ratio.max() <= 1.0, (f"layer {l} sequence {b} row {idx[at[0]]} head {at[1]} dim {at[2]}: got {got[at]} "
                                        f"want {want[at]} tol {tol[at]}")
    rest = batch.outside()
    if len(rest):
        assert bool((out[:, torch.from_numpy(rest).cuda()] == 7.0).all()), "rows of no sequence were written"
    return worst
