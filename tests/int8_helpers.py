"""Batches of packed sequences over int8 caches for the GPU tests (test infrastructure)."""

import numpy as np
import torch

from oracle import int8 as oracle
from tests.packed_helpers import host


class Int8Batch:
    """Sequences with `lens` new tokens over `ctxs` cached ones, in an int8 cache of pages in random order.  Pages and rows that no
    sequence has hold integers of 127, and pages that none has the scales `poison`."""

    def __init__(self, lens, ctxs, heads=(4, 2, 64), layers=1, windows=None, seed=0, lead=0, tail=0, poison=float("nan"), spare_pages=3,
                 spread=0.4, max_pages=None):
        from paper_2607_14431_amd import kvg
        self.kvg, self.heads, self.layers, self.windows = kvg, heads, layers, windows
        self.lens, self.ctxs = list(lens), list(ctxs)
        Hq, Hkv, D = heads
        rng = np.random.default_rng(seed)
        B = len(lens)
        self.max_pages = max_pages or max(-(-max(c + n, 1) // 16) for c, n in zip(ctxs, lens))
        n_pages = B * self.max_pages + spare_pages
        self.table = rng.permutation(n_pages)[:B * self.max_pages].reshape(B, self.max_pages).astype(np.int32)
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        known = np.zeros((n_pages, 16), dtype=bool)
        for b in range(B):
            for t in range(self.ctxs[b] + self.lens[b]):
                known[self.table[b, t // 16], t % 16] = True
        mine = torch.from_numpy(known).cuda()
        pools, scales = [], []
        for _ in range(2):
            x = torch.empty((layers, n_pages, Hkv, 16, D), dtype=torch.float32, device="cuda").normal_(0.0, 34.0, generator=self.gen)
            x = x.round_().clamp_(-127, 127).masked_fill_(~mine[None, :, None, :, None], 127.0)
            pools.append(x.to(torch.int8))
            s = torch.empty((layers, n_pages, Hkv), device="cuda").normal_(0.0, spread, generator=self.gen).exp_().div_(34.0)
            scales.append(s.masked_fill_(~mine.any(1)[None, :, None], poison))
        self.cache = kvg.Int8Cache(*pools, *scales, Hq, windows)
        self.cu = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int32) + lead
        self.tokens = int(self.cu[-1]) + tail
        self.start = rng.integers(0, 5000, B).astype(np.int64)
        self.seqs = kvg.Seqs(torch.from_numpy(self.table).cuda(), torch.tensor(self.ctxs, dtype=torch.int32, device="cuda"),
                             torch.from_numpy(self.start).cuda(), max(self.ctxs))
        self.packed = kvg.Packed(torch.from_numpy(self.cu).cuda(), self.tokens, max(self.lens))

    def rows(self, heads, sigma=1.0, wide=0):
        """Random bf16 rows [layers][tokens][heads][D]; wide > 0: a view into rows `wide` heads wider."""
        x = torch.empty((self.layers, self.tokens, heads + wide, self.heads[2]), dtype=torch.float32, device="cuda")
        x = x.normal_(0.0, sigma, generator=self.gen).to(torch.bfloat16)
        return x[:, :, wide // 2:wide // 2 + heads] if wide else x

    def workspace(self):
        return self.kvg.int8_attn_workspace(self.cache, self.seqs, self.packed, self.layers)

    def attend(self, q, scale, out=None, ws=None):
        if out is None:
            out = torch.full((self.layers, self.tokens, self.heads[0], self.heads[2]), 7.0, dtype=torch.bfloat16, device="cuda")
        self.kvg.kvg_int8_attn(self.cache, self.seqs, self.packed, 0, self.layers, q, scale, out,
                               self.workspace() if ws is None else ws)
        return out

    def cached(self, l, b, n=None):
        """Sequence b's integers [S][Hkv][D] and scales [S][Hkv] of keys, then of values, in layer l."""
        n = self.ctxs[b] + self.lens[b] if n is None else n
        pages = torch.from_numpy(self.table[b, :-(-n // 16)].astype(np.int64)).cuda()
        res = []
        for pool, scale in ((self.cache.k_pool, self.cache.k_scale), (self.cache.v_pool, self.cache.v_scale)):
            res.append(host(pool[l][pages]).transpose(0, 2, 1, 3).reshape(-1, *self.heads[1:])[:n])
            res.append(np.repeat(host(scale[l][pages]), 16, axis=0)[:n])
        return res

    def outside(self):
        """Packed rows that belong to no sequence."""
        mine = np.zeros(self.tokens, dtype=bool)
        for b, n in enumerate(self.lens):
            mine[self.cu[b]:self.cu[b] + n] = True
        return np.flatnonzero(~mine)


def check(batch, q, out, scale, rows_of=lambda n: range(n)):
    """Every sequence's rows against the oracle; rows of no sequence keep the fill value 7."""
    worst = 0.0
    for l in range(batch.layers):
        w = batch.windows[l] if batch.windows else 0
        for b, n in enumerate(batch.lens):
            idx = np.array(sorted(set(i for i in rows_of(n) if 0 <= i < n)), dtype=np.int64)
            if len(idx) == 0:
                continue
            r = torch.from_numpy(idx + int(batch.cu[b])).cuda()
            want, tol = oracle.attend(host(q[l][r]), idx + batch.ctxs[b], *batch.cached(l, b), scale, w)
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
