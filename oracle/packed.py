"""Scaled and partial rotary embeddings, head norms and attention of packed sequences, oracle side (test
infrastructure only).  fp64 throughout; the definitions are those of include/kvg.h.

Scaled rotaries: position interpolation divides every frequency by the factor; the base form changes the base so that the
slowest frequency is interpolated and the fastest stays; the rotations and index forms keep the
frequencies of many turns over the original context, interpolate those of few, and ramp between (by the number
of turns, or linearly over the index)."""

from __future__ import annotations

import math

import numpy as np


def frequencies(dim: int, base: float, scaling: str = "plain", factor: float = 1.0, original_len: float = 0.0,
                fast: float = 0.0, slow: float = 0.0) -> np.ndarray:
    """theta_i, i in [0, dim / 2)."""
    i = np.arange(dim // 2, dtype=np.float64)
    if scaling == "base":
        return np.exp(-2.0 * i / dim * (math.log(base) + dim / (dim - 2.0) * math.log(factor)))
    theta = np.exp(-2.0 * i / dim * math.log(base))
    if scaling == "plain":
        return theta
    if scaling == "linear":
        return theta / factor
    if scaling == "rotations":
        turns = original_len / (2 * math.pi / theta)
        interpolated = 1.0 - np.clip((turns - slow) / (fast - slow), 0.0, 1.0)
    elif scaling == "index":
        # the index whose frequency makes n turns over the original context, as a real number
        at = lambda n: dim / 2 * math.log(original_len / (2 * math.pi * n)) / math.log(base)  # noqa: E731
        lo, hi = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), dim - 1)
        interpolated = np.clip((i - lo) / (hi - lo if hi - lo >= 0.001 else 0.001), 0.0, 1.0)
    else:
        raise ValueError(scaling)
    return theta * (1.0 - interpolated) + theta * interpolated / factor


def pair_index(dim: int, pairing: str):
    a = np.arange(dim // 2)
    return (a, a + dim // 2) if pairing == "half" else (2 * a, 2 * a + 1)


def rotate(x: np.ndarray, pos: np.ndarray, theta: np.ndarray, pairing: str, amplitude: float = 1.0) -> np.ndarray:
    """x[..., T, H, D]: the first 2 len(theta) components of each head rotated by pos[T] * theta."""
    ia, ib = pair_index(2 * len(theta), pairing)
    phi = np.asarray(pos, dtype=np.float64)[:, None, None] * theta
    c, s = amplitude * np.cos(phi), amplitude * np.sin(phi)
    out = np.array(x, dtype=np.float64)
    out[..., ia] = x[..., ia] * c - x[..., ib] * s
    out[..., ib] = x[..., ia] * s + x[..., ib] * c
    return out


def axis_of_pairs(pairs, order: str) -> np.ndarray:
    """The axis of each pair: contiguous sections, or in turn until an axis has had its pairs."""
    if order == "sections":
        return np.repeat(np.arange(len(pairs)), pairs)
    # pair j of axis k comes in turn j, after that turn's pairs of the axes before k
    turns = sorted((j, k) for k, n in enumerate(pairs) for j in range(n))
    return np.array([k for _, k in turns])


def axes_frequencies(pairs, base, own: bool, **scaling) -> np.ndarray:
    """theta of each pair: the whole rotary's, or every axis' own (sections)."""
    if not own:
        return frequencies(2 * sum(pairs), base, **scaling)
    return np.concatenate([frequencies(2 * n, base, **scaling) for n in pairs])


def rotate_axes(x, pos, theta, axis, pairing, amplitude=1.0) -> np.ndarray:
    """x[..., T, H, D]: pair i turned by pos[axis[i]][T] * theta[i]."""
    out = np.array(x, dtype=np.float64)
    ia, ib = pair_index(2 * len(theta), pairing)
    for i, t in enumerate(theta):
        phi = np.asarray(pos[axis[i]], dtype=np.float64)[:, None] * t
        z = (x[..., ia[i]] + 1j * x[..., ib[i]]) * (amplitude * np.exp(1j * phi))
        out[..., ia[i]], out[..., ib[i]] = z.real, z.imag
    return out


def rms_norm(x: np.ndarray, weight: np.ndarray, eps: float, offset: float) -> np.ndarray:
    return x / np.sqrt(np.mean(np.square(x), axis=-1, keepdims=True) + eps) * (weight + offset)


def attend_bounds(q, index, k, v, scale, window=0):
    """Attention of rows q [T][Hq][D] at logical indices `index` over keys [S][Hkv][D], as oracle.attention.attend, and
    what an error bound needs, each [T][Hq][D]: (out, spread, mass, score) with weights w_j
      spread = sum_j w_j |v_j - out|, mass = sum_j w_j |v_j|, score = sum_j w_j (sum_d |q_d k_jd|) scale |v_j - out|."""
    T, Hq, D = q.shape
    group = Hq // k.shape[1]
    j = np.arange(k.shape[0])[None, :]
    hidden = j > index[:, None]
    if window > 0:
        hidden |= j <= index[:, None] - window
    res = [np.empty((T, Hq, D)) for _ in range(4)]
    for h in range(Hq):
        kh, vh = k[:, h // group], v[:, h // group]
        s = np.where(hidden, -np.inf, q[:, h] @ kh.T * scale)
        w = np.exp(s - s.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        size = np.abs(q[:, h]) @ np.abs(kh).T * scale
        out = w @ np.where(np.isfinite(vh), vh, 0.0)
        for t in range(T):
            seen = ~hidden[t]
            away = np.abs(vh[seen] - out[t])
            res[1][t, h] = w[t, seen] @ away
            res[2][t, h] = w[t, seen] @ np.abs(vh[seen])
            res[3][t, h] = (w[t, seen] * size[t, seen]) @ away
        res[0][:, h] = out
    return res
