"""Payloads that kernels cannot read or write, refused by the binding before anything is launched (no GPU needed)."""

import pytest
import torch

kvg = pytest.importorskip("paper_2607_14431_amd.kvg", reason="libkvg.so not built")


def _calls():
    """name: (bytes of a payload, call with one)"""
    table = torch.zeros(2, dtype=torch.int32)
    pool, scale = torch.zeros(1, 2, 2, 16, 64), torch.zeros(1, 2, 2)
    c = kvg.Cache(pool.to(torch.bfloat16), pool.to(torch.bfloat16), 4)
    c8 = kvg.Int8Cache(pool.to(torch.int8), pool.to(torch.int8), scale, scale.clone(), 4)
    h, h8 = kvg.kvg_artifact_header_init(c, 20, 0, kvg.rope()), kvg.kvg_int8_header_init(c8, 20, 0)
    return {"deposit": (h.payload_bytes, lambda p: kvg.kvg_deposit(c, table, 0, 20, p)),
            "graft": (h.payload_bytes, lambda p: kvg.kvg_graft(c, h, p, table, 0, 0)),
            "int8_deposit": (h8.payload_bytes, lambda p: kvg.kvg_int8_deposit(c8, table, 0, 20, p)),
            "int8_graft": (h8.payload_bytes, lambda p: kvg.kvg_int8_graft(c8, h8, p, table, 0, 0))}


@pytest.mark.parametrize("name", ["deposit", "graft", "int8_deposit", "int8_graft"])
def test_payloads(monkeypatch, name):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)        # the cache and its table pass as the current device's
    n, call = _calls()[name]
    for bad, words in ((torch.zeros(n, dtype=torch.uint8), "pinned host memory"),        # pageable host memory
                       (torch.zeros(n - 1, dtype=torch.uint8), "bytes"),
                       (torch.zeros(2 * n, dtype=torch.uint8)[::2], "contiguous"),
                       (torch.zeros(1, dtype=torch.uint8).expand(n), "contiguous")):
        with pytest.raises(ValueError, match=words):
            call(bad)


@pytest.mark.parametrize("name", ["int8_deposit", "int8_graft"])
def test_payloads_of_another_device(monkeypatch, name):
    """The payload is among the tensors whose device is checked."""
    n, call = _calls()[name]
    seen = []

    def check(*tensors):
        seen.extend(tensors)
        raise ValueError("stop before the launch")

    monkeypatch.setattr(kvg, "_on_current_device", check)
    payload = torch.zeros(n, dtype=torch.uint8)
    monkeypatch.setattr(kvg, "_payload_ok", lambda p, *_: p)             # as of a device
    with pytest.raises(ValueError, match="stop"):
        call(payload)
    assert any(t is payload for t in seen)
