"""Sampling: refusals on the host (no GPU needed), the binding's checks, and the oracle."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import sampling as oracle

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")

INVAL, SHAPE, ALIGN, WORKSPACE = -1, -2, -6, -9


def _sample(logits=0x1000, stride=0, rows=2, vocab=100, sampling=True, temperature=0x2000, uniform=0x3000, tokens=0x4000, ws=0x5000,
            ws_bytes=None):
    if ws_bytes is None:
        ws_bytes = kvg.raw_call("kvg_sample_workspace_bytes", rows, vocab)
    s = kvg.kvg_sampling(temperature, None, None, None)
    return kvg.raw_call("kvg_sample", logits, stride, rows, vocab, ctypes.byref(s) if sampling else None, uniform, tokens, None, ws, ws_bytes,
                        None)


def test_refusals():
    assert _sample(rows=0) == 0 and _sample(rows=0, logits=None, uniform=None, tokens=None, temperature=None) == 0
    assert _sample(rows=-1, ws_bytes=1 << 20) == INVAL and _sample(vocab=0, ws_bytes=1 << 20) == INVAL and _sample(sampling=False) == INVAL
    assert _sample(stride=99) == INVAL and _sample(stride=-200) == INVAL
    assert _sample(logits=None) == INVAL and _sample(uniform=None) == INVAL and _sample(tokens=None) == INVAL
    assert _sample(temperature=None) == INVAL
    assert _sample(vocab=(1 << 24) + 1, ws_bytes=1 << 30) == SHAPE and _sample(rows=65536, ws_bytes=1 << 40) == SHAPE
    assert _sample(ws=None) == WORKSPACE and _sample(ws_bytes=0) == WORKSPACE and _sample(ws=0x5008) == ALIGN
    size = lambda r, v: kvg.raw_call("kvg_sample_workspace_bytes", r, v)  # noqa: E731
    assert size(-1, 5) == 0 and size(5, 0) == 0 and size(5, (1 << 24) + 1) == 0 and size(65536, 5) == 0
    assert size(1, 1) > 0 and size(65535, 1 << 24) > 0


def test_binding_checks():
    f, d, i = torch.zeros(3), torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.int32)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    x = torch.zeros(3, 10)
    for args, kw in (((x.double(), f, d, i, ws), {}), ((x.t().contiguous().t(), f, d, i, ws), {}), ((x[:1].expand(3, 10), f, d, i, ws), {}),
                     ((x, d, d, i, ws), {}), ((x, f, f, i, ws), {}), ((x, f, d, f, ws), {}), ((x, f[:2], d, i, ws), {}),
                     ((x, f, d, i, ws), dict(top_k=f)), ((x, f, d, i, ws), dict(top_p=d)), ((x, f, d, i, ws), dict(min_p=torch.zeros(6)[::2])),
                     ((x, f, d, i, ws), dict(logprobs=d)), ((x, f, d, i, ws[::2]), {})):
        with pytest.raises(ValueError):
            kvg.kvg_sample(*args, **kw)


def test_oracle():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3], dtype=np.float64)).astype(np.float32)
    token = lambda u, **kw: oracle.sample(l, 1.0, u, **kw)[0]  # noqa: E731
    assert [token(u) for u in (0.0, 0.05, 0.2, 0.6, 0.8, 1.5)] == [0, 0, 1, 2, 3, 3]
    assert [token(u, top_k=2) for u in (0.0, 0.5, 0.6)] == [1, 1, 3]                 # 0.4 and 0.3 of 0.7
    assert token(0.99, top_p=0.35) == 1 and token(0.99, top_p=0.45) == 3 and token(0.99, top_p=0.0) == 1
    assert token(0.99, min_p=0.6) == 3 and token(0.0, min_p=0.6) == 1 and token(0.3, min_p=9.0) == 1
    assert token(0.5, top_k=3, top_p=0.8) == 2 and token(0.9, top_k=3, top_p=0.7) == 3    # 0.4 + 0.3 of 0.9 is 0.78: all three, two
    assert abs(oracle.sample(l, 1.0, 0.3, top_k=2)[1] - math.log(4 / 7)) < 1e-6
    assert abs(oracle.sample(l, 0.5, 0.3)[1] - math.log(0.16 / 0.30)) < 1e-6
    assert oracle.sample(np.array([1, 3, 3, 2], dtype=np.float32), 0.0, 0.9)[:2] == (1, 0.0)
    assert oracle.sample(np.array([1, 3, 3, 3], dtype=np.float32), 1.0, 0.9, top_k=2)[0] == 2    # ties: the lowest indices
    assert oracle.sample(np.array([-math.inf, -math.inf], dtype=np.float32), 1.0, 0.5)[0] == -1
