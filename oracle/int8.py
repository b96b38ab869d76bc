"""8-bit integer caches with a scale for each page and KV head, oracle side (test infrastructure only).  fp64 throughout; the
definitions are those of include/kvg.h."""

from __future__ import annotations

import numpy as np

PAGE = 16
U = 2.0 ** -24


def append_page(held: np.ndarray, before: float, new: np.ndarray):
    """(integers of the held rows, integers of the new ones, scale) of one page and KV head: held [h][D] integers at scale
    `before` (not read when h is 0), new [n][D] values."""
    scale = np.abs(new).max() / 127.0 if new.size else 0.0
    if len(held):
        scale = max(scale, before)
    if scale == 0.0:
        return np.zeros_like(held), np.zeros(new.shape), 0.0
    return np.rint(held * (before / scale)) if len(held) else held, np.rint(new / scale), scale


def attend(q, index, kn, ks, vn, vs, scale, window=0):
    """(want, tol) of attention rows q [T][Hq][D] at logical indices `index` over cached integers kn, vn [S][Hkv][D] with
    scales ks, vs [S][Hkv] of their pages, each [T][Hq][D].

    tol: the query is rounded to multiples of 2^(e - 14), 2^e > max |q| >= 2^(e - 1), so each component is off by at most 2^-14 max
    |q|; the integer products are exact; the scores' conversion, scales and difference to the reference round a few times
    each (8 u of the score's size and 24 u), the exponential 2 u.  A score off by d moves a row by w d |v - out|.  A weight times
    its scale rounds to fp16, in units in which the largest of its segment of keys is above 2^6: 2^-11 of itself, or below 2^-14 of
    them half of fp16's last step, 2^-25, which is 2^-31 of the row's largest; the sum of
    the weights does not, so it moves a row by that part of w |v|.  Sums of n terms add n u.  The result rounds to bf16."""
    T, Hq, D = q.shape
    S, Hkv = ks.shape
    group = Hq // Hkv
    j = np.arange(S)[None, :]
    hidden = j > index[:, None]
    if window > 0:
        hidden |= j <= index[:, None] - window
    want, tol = np.empty((T, Hq, D)), np.empty((T, Hq, D))
    for h in range(Hq):
        g = h // group
        k, v = kn[:, g] * ks[:, g, None], vn[:, g] * vs[:, g, None]
        s = q[:, h] @ k.T * scale
        size = np.abs(q[:, h]) @ np.abs(k).T * scale
        off = 2.0 ** -14 * np.abs(q[:, h]).max(axis=1)[:, None] * np.abs(k).sum(axis=1)[None, :] * scale + 8 * U * size + 26 * U
        s = np.where(hidden, -np.inf, s)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        for t in range(T):
            seen = ~hidden[t]
            wt, vt = w[t, seen], v[seen]
            out = wt @ vt
            mass = wt @ np.abs(vt)
            top = (wt * vs[seen, g]).max()
            moved = (wt * off[t, seen]) @ np.abs(vt - out)
            small = 2.0 ** -31 * top * np.abs(vn[seen, g]).sum(axis=0)
            err = 1.02 * moved + (2.0 ** -11 + 4 * U) * mass + small + (seen.sum() + 8) * U * (mass + np.abs(out))
            want[t, h] = out
            tol[t, h] = err + 2.0 ** -8 * (np.abs(out) + err) + 1e-37
    return want, tol
