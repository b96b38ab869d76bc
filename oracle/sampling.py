"""Sampling from logits, oracle side (test infrastructure only): the definition of include/kvg.h in extended precision."""

from __future__ import annotations

import math

import numpy as np


def sample(logits, temperature, u, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, margin) of one row of fp32 logits.  margin: how far, in units of the row's largest weight, the closest of
    the choices made (the share top_p, the bound min_p, the random number) is from being made otherwise."""
    l = np.asarray(logits, dtype=np.float32)
    nan = float("nan")
    if np.isnan(l).any() or np.isposinf(l).any() or not np.isfinite(l).any():
        return -1, nan, math.inf
    if not (0 <= temperature < math.inf) or any(math.isnan(x) for x in (u, top_p, min_p)):
        return -1, nan, math.inf
    order = np.lexsort((np.arange(len(l)), -l.astype(np.float64)))      # by value, then by index
    if temperature == 0:
        return int(order[0]), 0.0, math.inf
    with np.errstate(over="ignore", invalid="ignore"):
        y = (l.astype(np.longdouble) - np.longdouble(l[order[0]])) / np.longdouble(temperature)
    e = np.exp(y)
    margin = math.inf
    n = len(l) if top_k <= 0 else min(len(l), top_k)
    if top_p < 1:
        c = np.cumsum(e[order[:n]])
        share = max(np.longdouble(top_p), 0) * c[-1]
        m = next(i for i in range(n) if c[i] >= share)
        if share > 0:
            margin = min(margin, float(np.abs(c - share).min()))
        n = m + 1
    if min_p > 0:
        bound = min(min_p, 1.0)
        margin = min([margin] + [float(abs(x - bound)) for x in e[order[1:]] if x != 1])
        while n > 1 and e[order[n - 1]] < bound:
            n -= 1
    keep = np.sort(order[:n])
    c = np.cumsum(e[keep])
    at = min(max(np.longdouble(u), 0), 1) * c[-1]
    i = next((i for i in range(n) if c[i] > at), None)
    if i is None:                                    # u >= 1: the last one with a weight
        i = max(j for j in range(n) if e[keep[j]] > 0)
    if 0 < u < 1:
        margin = min(margin, float(np.abs(c - at).min()))
    return int(keep[i]), float(y[keep[i]] - np.log(c[-1])), margin
