"""Python binding of libkvg.so: same names as the C ABI (include/kvg.h), argument
marshalling only.  Every step runs in the library's HIP kernels; torch supplies device
memory and the stream.  Importing this module without the built library raises.
"""

from __future__ import annotations

import ctypes
import dataclasses
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvg.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_14431_amd.build` "
                      "(there is no fallback path)")
_lib = ctypes.CDLL(LIB_PATH)

KVG_F32, KVG_BF16, KVG_FP8_E4M3, KVG_INT8 = 0, 1, 2, 3
KVG_ROPE_HALF, KVG_ROPE_INTERLEAVED, KVG_ROPE_OTHER = 0, 1, 2
KVG_GRAFT_ALLOW_RELOCATE = 1
KVG_ROTARY_PLAIN, KVG_ROTARY_LINEAR, KVG_ROTARY_BASE, KVG_ROTARY_ROTATIONS, KVG_ROTARY_INDEX = range(5)
KVG_AXES_SECTIONS, KVG_AXES_TURNS = 0, 1
KVG_MAX_AXES = 4
KVG_ARTIFACT_MAGIC = 0x4147564B
KVG_ARTIFACT_VERSION = 2

STATUS = {
    0: "KVG_OK", -1: "KVG_E_INVAL", -2: "KVG_E_SHAPE", -3: "KVG_E_DTYPE", -4: "KVG_E_POSITION",
    -5: "KVG_E_CAPACITY", -6: "KVG_E_ALIGN", -7: "KVG_E_CORRUPT", -8: "KVG_E_HIP", -9: "KVG_E_WORKSPACE",
}


class KvgError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        self.name = STATUS.get(status, str(status))
        super().__init__(f"{where}: {self.name} ({kvg_status_str(status)})")


class kvg_rope(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("pairing", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class kvg_cache(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_pages", ctypes.c_int64), ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("layer_window", ctypes.POINTER(ctypes.c_int32))]


class kvg_int8_cache(ctypes.Structure):
    _fields_ = [("pages", kvg_cache), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class kvg_seqs(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_ctx_len", ctypes.c_int32),
                ("shared_tokens", ctypes.c_int32), ("block_tables", ctypes.c_void_p), ("ctx_lens", ctypes.c_void_p),
                ("start_pos", ctypes.c_void_p)]


class kvg_rotary(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("factor", ctypes.c_double), ("original_len", ctypes.c_double),
                ("fast", ctypes.c_double), ("slow", ctypes.c_double), ("amplitude", ctypes.c_double),
                ("pairing", ctypes.c_int32), ("scaling", ctypes.c_int32), ("rotary_dim", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class kvg_head_norm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("weight_offset", ctypes.c_float)]


class kvg_packed(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int32), ("max_len", ctypes.c_int32), ("cu_tokens", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


class kvg_axes(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("n_axes", ctypes.c_int32), ("order", ctypes.c_int32),
                ("own_frequencies", ctypes.c_int32), ("reserved", ctypes.c_int32), ("pairs", ctypes.c_int32 * 4)]


class kvg_sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


class kvg_artifact_hdr(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_uint32), ("version", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("own_pos", ctypes.c_int64),
                ("rope_base", ctypes.c_double), ("rope_pairing", ctypes.c_int32),
                ("digest_leaf_bytes", ctypes.c_uint32), ("payload_bytes", ctypes.c_uint64),
                ("digest", ctypes.c_uint8 * 32)]


_P = ctypes.POINTER
_vp, _i32, _i64, _sz, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
_u64 = ctypes.c_uint64

_SIGS = {
    "kvg_version": (ctypes.c_char_p, []),
    "kvg_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "kvg_payload_bytes": (_sz, [_P(kvg_cache), _i32]),
    "kvg_artifact_header_init": (ctypes.c_int, [_P(kvg_cache), _i32, _i64, _P(kvg_rope), _P(kvg_artifact_hdr)]),
    "kvg_artifact_digest_workspace_bytes": (_sz, [_P(kvg_artifact_hdr)]),
    "kvg_artifact_seal": (ctypes.c_int, [_P(kvg_artifact_hdr), _vp, _vp, _sz, _vp]),
    "kvg_artifact_verify": (ctypes.c_int, [_P(kvg_artifact_hdr), _vp, _vp, _sz, _vp]),
    "kvg_append": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_rope), _i32, _i32, _i32, _vp, _vp, _vp]),
    "kvg_deposit": (ctypes.c_int, [_P(kvg_cache), _vp, _i32, _i32, _i32, _vp, _vp]),
    "kvg_graft": (ctypes.c_int, [_P(kvg_cache), _P(kvg_artifact_hdr), _vp, _vp, _i32, _i32, _i64, _i32, _vp]),
    "kvg_prefill_workspace_bytes": (_sz, [_P(kvg_cache), _P(kvg_seqs), _i32, _i32]),
    "kvg_prefill_attn": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_rope), _i32, _i32, _i32, _vp, _vp,
                                        _vp, _f32, _vp, _vp, _sz, _vp]),
    "kvg_decode_workspace_bytes": (_sz, [_P(kvg_cache), _P(kvg_seqs), _i32]),
    "kvg_decode_attn": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_rope), _i32, _i32, _vp, _vp, _vp,
                                       _f32, _vp, _vp, _sz, _vp]),
    "kvg_decode_attn_noalloc": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_rope), _i32, _i32, _vp, _vp, _vp,
                                               _f32, _vp, _vp]),
    "kvg_rotary_frequencies": (ctypes.c_int, [_P(kvg_rotary), _i32, _P(ctypes.c_double)]),
    "kvg_artifact_header_init_rotary": (ctypes.c_int, [_P(kvg_cache), _i32, _i64, _P(kvg_rotary), _P(kvg_artifact_hdr)]),
    "kvg_rotate": (ctypes.c_int, [_P(kvg_rotary), _i32, _i32, _i32, _i32, _vp, _vp, _i64, _vp, _i64, _vp]),
    "kvg_norm_append": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_packed), _P(kvg_rotary), _P(kvg_head_norm),
                                       _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "kvg_artifact_header_init_axes": (ctypes.c_int, [_P(kvg_cache), _i32, _i64, _P(kvg_rotary), _P(kvg_axes), _P(kvg_artifact_hdr)]),
    "kvg_rotate_axes": (ctypes.c_int, [_P(kvg_rotary), _P(kvg_axes), _i32, _i32, _i32, _i32, _vp, _i64, _vp, _i64, _vp]),
    "kvg_norm_append_axes": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_packed), _P(kvg_rotary), _P(kvg_axes),
                                            _P(kvg_head_norm), _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "kvg_packed_attn_workspace_bytes": (_sz, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_packed), _i32]),
    "kvg_packed_attn": (ctypes.c_int, [_P(kvg_cache), _P(kvg_seqs), _P(kvg_packed), _i32, _i32, _vp, _f32, _vp, _vp, _sz,
                                       _vp]),
    "kvg_int8_append": (ctypes.c_int, [_P(kvg_int8_cache), _P(kvg_seqs), _P(kvg_packed), _P(kvg_rotary), _P(kvg_axes),
                                       _P(kvg_head_norm), _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "kvg_int8_attn_workspace_bytes": (_sz, [_P(kvg_int8_cache), _P(kvg_seqs), _P(kvg_packed), _i32]),
    "kvg_int8_attn": (ctypes.c_int, [_P(kvg_int8_cache), _P(kvg_seqs), _P(kvg_packed), _i32, _i32, _vp, _f32, _vp, _vp, _sz,
                                     _vp]),
    "kvg_int8_payload_bytes": (_sz, [_P(kvg_int8_cache), _i32]),
    "kvg_int8_header_init": (ctypes.c_int, [_P(kvg_int8_cache), _i32, _i64, _P(kvg_artifact_hdr)]),
    "kvg_int8_deposit": (ctypes.c_int, [_P(kvg_int8_cache), _vp, _i32, _i32, _i32, _vp, _vp]),
    "kvg_int8_graft": (ctypes.c_int, [_P(kvg_int8_cache), _P(kvg_artifact_hdr), _vp, _vp, _i32, _i32, _i64, _vp]),
    "kvg_leaf_digests": (ctypes.c_int, [_vp, _u64, ctypes.c_uint32, _vp, _vp]),
    "kvg_merkle_workspace_bytes": (_sz, [_u64]),
    "kvg_merkle_root": (ctypes.c_int, [_vp, _u64, _vp, _vp, _sz, _vp]),
    "kvg_dedup_workspace_bytes": (_sz, [_u64]),
    "kvg_dedup_map": (ctypes.c_int, [_vp, _u64, _vp, _vp, _vp, _sz, _vp]),
    "kvg_logits_packed_bytes": (_sz, [_i32, _i32]),
    "kvg_logits_pack": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp]),
    "kvg_logits_workspace_bytes": (_sz, [_i32, _i32]),
    "kvg_logits": (ctypes.c_int, [_vp, _i32, _i32, _vp, _i32, _f32, _vp, _vp, _sz, _vp]),
    "kvg_sample_workspace_bytes": (_sz, [_i32, _i32]),
    "kvg_sample": (ctypes.c_int, [_vp, _i64, _i32, _i32, _P(kvg_sampling), _vp, _vp, _vp, _vp, _sz, _vp]),
    "kvg_logit_compare": (ctypes.c_int, [_vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

EXPORTED = tuple(_SIGS)


def kvg_version() -> str:
    return _lib.kvg_version().decode()


def kvg_status_str(status: int) -> str:
    return _lib.kvg_status_str(status).decode()


def _check(status: int, where: str):
    if status != 0:
        raise KvgError(status, where)


# Addresses go to the library as plain ints (its argument types convert them): a decode step's
# marshalling is a large part of a small call's time.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:
        # the current stream's handle, without the Stream object that torch.cuda.current_stream() makes
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def rope(base: float = 10000.0, pairing: int = KVG_ROPE_HALF) -> kvg_rope:
    return kvg_rope(base, pairing, 0)


_DTYPE_CODE = {torch.float32: KVG_F32, torch.bfloat16: KVG_BF16, torch.float8_e4m3fn: KVG_FP8_E4M3}


def _pages_struct(k: torch.Tensor, v: torch.Tensor, n_q_heads: int, code: int, windows) -> kvg_cache:
    """The struct of two paged pools."""
    shape = k.shape
    if not (k.is_contiguous() and v.is_contiguous() and shape == v.shape and k.dtype == v.dtype):
        raise ValueError("pools: contiguous, of one shape and type")
    n_layers, n_pages, n_kv_heads, page_size, head_dim = shape
    c = kvg_cache(n_layers, n_q_heads, n_kv_heads, head_dim, page_size, code, n_pages, k.data_ptr(), v.data_ptr(), None)
    if windows is not None and any(windows):
        if len(windows) != n_layers:
            raise ValueError("windows: one per layer")
        arr = (ctypes.c_int32 * len(windows))(*windows)
        c.layer_window = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
        c._windows_keepalive = arr        # the struct holds a raw pointer into this array
    return c


@dataclasses.dataclass
class Cache:
    """Paged pools [n_layers][n_pages][n_kv_heads][page_size][head_dim] (torch tensors)."""
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    n_q_heads: int
    windows: tuple | None = None       # per-layer sliding window (0 = full causal), or None

    @staticmethod
    def allocate(n_layers, n_pages, n_q_heads, n_kv_heads, head_dim, dtype: torch.dtype, device="cuda",
                 page_size=16, windows=None):
        shape = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
        if windows is not None:
            windows = tuple(int(x) for x in windows)
            if len(windows) != n_layers:
                raise ValueError("windows: one per layer")
        return Cache(torch.empty(shape, dtype=dtype, device=device),
                     torch.empty(shape, dtype=dtype, device=device), n_q_heads, windows)

    @property
    def n_layers(self):
        return self.k_pool.shape[0]

    @property
    def n_pages(self):
        return self.k_pool.shape[1]

    @property
    def n_kv_heads(self):
        return self.k_pool.shape[2]

    @property
    def page_size(self):
        return self.k_pool.shape[3]

    @property
    def head_dim(self):
        return self.k_pool.shape[4]

    @property
    def kvg_dtype(self):
        return _DTYPE_CODE[self.k_pool.dtype]

    @property
    def raw_dtype(self) -> torch.dtype:
        """dtype of the raw q/k/v this cache takes (bf16 for an fp8 cache)."""
        dtype = self.k_pool.dtype
        return torch.bfloat16 if dtype is torch.float8_e4m3fn else dtype

    def struct(self) -> kvg_cache:
        return _pages_struct(self.k_pool, self.v_pool, self.n_q_heads, _DTYPE_CODE[self.k_pool.dtype], self.windows)


@dataclasses.dataclass
class Seqs:
    """Block tables [batch][max_pages] int32, ctx_lens [batch] int32, start_pos [batch] int64 (device);
    shared_tokens: leading tokens whose table entries all sequences share (0 = none)."""
    block_tables: torch.Tensor
    ctx_lens: torch.Tensor
    start_pos: torch.Tensor
    max_ctx_len: int
    shared_tokens: int = 0      # leading tokens every sequence's table shares (see kvg_seqs in kvg.h)

    def struct(self) -> kvg_seqs:
        bt, ctx, pos = self.block_tables, self.ctx_lens, self.start_pos
        shape = bt.shape
        if not (bt.dtype is torch.int32 and bt.is_contiguous() and len(shape) == 2 and ctx.dtype is torch.int32 and
                pos.dtype is torch.int64):
            raise ValueError("block_tables: int32 [batch][max_pages], contiguous; ctx_lens: int32; start_pos: int64")
        if not (ctx.numel() >= shape[0] <= pos.numel() and ctx.is_contiguous() and pos.is_contiguous()):
            raise ValueError("ctx_lens, start_pos: [batch], contiguous")
        return kvg_seqs(shape[0], shape[1], self.max_ctx_len, self.shared_tokens, bt.data_ptr(), ctx.data_ptr(),
                        pos.data_ptr())


def kvg_payload_bytes(cache: Cache, n_tokens: int) -> int:
    return _lib.kvg_payload_bytes(ctypes.byref(cache.struct()), n_tokens)


def kvg_artifact_header_init(cache: Cache, n_tokens: int, own_pos: int, rp: kvg_rope) -> kvg_artifact_hdr:
    hdr = kvg_artifact_hdr()
    _check(_lib.kvg_artifact_header_init(ctypes.byref(cache.struct()), n_tokens, own_pos, ctypes.byref(rp),
                                         ctypes.byref(hdr)), "kvg_artifact_header_init")
    return hdr


def kvg_artifact_digest_workspace_bytes(hdr: kvg_artifact_hdr) -> int:
    return _lib.kvg_artifact_digest_workspace_bytes(ctypes.byref(hdr))


def _payload_ptr(payload):
    """Device address of a payload: a torch tensor, or an object with data_ptr() (pinned host
    memory exposed through its device address)."""
    return payload.data_ptr()


def _payload_ok(payload, nbytes: int, what: str):
    """Checks of a payload that kernels read or write: `nbytes` of dense bytes, in device or pinned host memory (what is not a torch tensor
    gives its own device address).  The tensor, if it is a device's."""
    if payload.nbytes < nbytes:
        raise ValueError(f"payload: {what}")
    if isinstance(payload, torch.Tensor):
        if not payload.is_contiguous():
            raise ValueError("payload: contiguous")
        if not payload.is_cuda and not payload.is_pinned():
            raise ValueError(f"payload: on the device or in pinned host memory, got {payload.device}")
        return payload if payload.is_cuda else None
    return None


def kvg_artifact_seal(hdr: kvg_artifact_hdr, payload, ws: torch.Tensor, stream=None):
    _check(_lib.kvg_artifact_seal(ctypes.byref(hdr), _payload_ptr(payload), _ptr(ws), ws.nbytes, _stream(stream)),
           "kvg_artifact_seal")


def kvg_artifact_verify(hdr: kvg_artifact_hdr, payload, ws: torch.Tensor, stream=None) -> int:
    """Status of the verification: 0 (KVG_OK) or KVG_E_CORRUPT (-7); other errors raise."""
    st = _lib.kvg_artifact_verify(ctypes.byref(hdr), _payload_ptr(payload), _ptr(ws), ws.nbytes, _stream(stream))
    if st not in (0, -7):
        raise KvgError(st, "kvg_artifact_verify")
    return st


def _raw_ok(cache: Cache, *raws):
    dtype = cache.raw_dtype
    for t in raws:
        if t.dtype is not dtype or not t.is_contiguous():
            raise ValueError("raw inputs: the cache's raw dtype, contiguous")


def kvg_append(cache: Cache, seqs: Seqs, rp: kvg_rope, layer0: int, n_layers: int, chunk_len: int,
               k_raw: torch.Tensor, v_raw: torch.Tensor, stream=None):
    _raw_ok(cache, k_raw, v_raw)
    _check(_lib.kvg_append(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), ctypes.byref(rp), layer0,
                           n_layers, chunk_len, _ptr(k_raw), _ptr(v_raw), _stream(stream)), "kvg_append")


def kvg_deposit(cache: Cache, block_table_row: torch.Tensor, first_token: int, n_tokens: int,
                payload: torch.Tensor, stream=None):
    _payload_ok(payload, kvg_payload_bytes(cache, n_tokens), "kvg_payload_bytes(cache, n_tokens) bytes")
    _check(_lib.kvg_deposit(ctypes.byref(cache.struct()), _ptr(block_table_row), block_table_row.numel(),
                            first_token, n_tokens, _ptr(payload), _stream(stream)), "kvg_deposit")


def kvg_graft(cache: Cache, hdr: kvg_artifact_hdr, payload: torch.Tensor, block_table_row: torch.Tensor,
              first_token: int, target_pos: int, flags: int = 0, stream=None):
    _payload_ok(payload, hdr.payload_bytes, "the header's payload_bytes")
    _check(_lib.kvg_graft(ctypes.byref(cache.struct()), ctypes.byref(hdr), _ptr(payload), _ptr(block_table_row),
                          block_table_row.numel(), first_token, target_pos, flags, _stream(stream)), "kvg_graft")


def kvg_prefill_workspace_bytes(cache: Cache, seqs: Seqs, n_layers: int, chunk_len: int) -> int:
    return _lib.kvg_prefill_workspace_bytes(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), n_layers,
                                            chunk_len)


def kvg_prefill_attn(cache: Cache, seqs: Seqs, rp: kvg_rope, layer0: int, n_layers: int, chunk_len: int,
                     q_raw, k_raw, v_raw, scale: float, out: torch.Tensor, ws: torch.Tensor, stream=None):
    _raw_ok(cache, q_raw, k_raw, v_raw)
    _check(_lib.kvg_prefill_attn(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), ctypes.byref(rp),
                                 layer0, n_layers, chunk_len, _ptr(q_raw), _ptr(k_raw), _ptr(v_raw), scale,
                                 _ptr(out), _ptr(ws), ws.nbytes, _stream(stream)), "kvg_prefill_attn")


def kvg_decode_workspace_bytes(cache: Cache, seqs: Seqs, n_layers: int) -> int:
    return _lib.kvg_decode_workspace_bytes(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), n_layers)


def decode_workspace(cache: Cache, seqs: Seqs, n_layers: int) -> torch.Tensor:
    """Scratch for kvg_decode_attn sized for `seqs` (covers any call with max_ctx_len no larger)."""
    return torch.empty(max(kvg_decode_workspace_bytes(cache, seqs, n_layers), 256), dtype=torch.uint8,
                       device=cache.k_pool.device)


def kvg_decode_attn(cache: Cache, seqs: Seqs, rp: kvg_rope, layer0: int, n_layers: int, q_raw, k_raw, v_raw,
                    scale: float, out: torch.Tensor, ws: torch.Tensor, stream=None):
    _raw_ok(cache, q_raw, k_raw, v_raw)
    _check(_lib.kvg_decode_attn(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), ctypes.byref(rp),
                                layer0, n_layers, _ptr(q_raw), _ptr(k_raw), _ptr(v_raw), scale, _ptr(out), _ptr(ws),
                                ws.nbytes, _stream(stream)), "kvg_decode_attn")


KVG_NOALLOC_SCRATCH_BYTES = 256 << 20


def kvg_decode_attn_noalloc(cache: Cache, seqs: Seqs, rp: kvg_rope, layer0: int, n_layers: int, q_raw, k_raw, v_raw,
                            scale: float, out: torch.Tensor, stream=None):
    """kvg_decode_attn on the library's own fixed workspace (no allocation by anyone)."""
    _raw_ok(cache, q_raw, k_raw, v_raw)
    _check(_lib.kvg_decode_attn_noalloc(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), ctypes.byref(rp),
                                        layer0, n_layers, _ptr(q_raw), _ptr(k_raw), _ptr(v_raw), scale, _ptr(out),
                                        _stream(stream)), "kvg_decode_attn_noalloc")


def rotary(base: float = 10000.0, pairing: int = KVG_ROPE_HALF, rotary_dim: int = 0, scaling: int = KVG_ROTARY_PLAIN,
           factor: float = 1.0, original_len: float = 0.0, fast: float = 0.0, slow: float = 0.0,
           amplitude: float = 1.0) -> kvg_rotary:
    """A rotary embedding: pairing, rotated part of the head (0: all of it), scaling with its parameters (kvg.h)."""
    return kvg_rotary(base, factor, original_len, fast, slow, amplitude, pairing, scaling, rotary_dim, 0)


@dataclasses.dataclass
class HeadNorm:
    """RMS norm of query and key heads: weights [n_layers][head_dim] of the raw dtype (None: not normed)."""
    q_weight: torch.Tensor | None
    k_weight: torch.Tensor | None
    eps: float
    weight_offset: float = 0.0       # 1 for weights stored less one

    def struct(self, cache: Cache, n_layers: int) -> kvg_head_norm:
        dtype, n = cache.raw_dtype, n_layers * cache.head_dim
        for w in (self.q_weight, self.k_weight):
            if w is not None and not (w.dtype is dtype and w.is_contiguous() and w.numel() == n):
                raise ValueError("norm weights: [n_layers][head_dim] of the cache's raw dtype, contiguous")
        return kvg_head_norm(_ptr(self.q_weight), _ptr(self.k_weight), self.eps, self.weight_offset)


@dataclasses.dataclass
class Packed:
    """New tokens of a batch, one sequence after the other: rows [cu_tokens[b], cu_tokens[b + 1]) (int32 [batch + 1],
    device) of tensors of n_tokens rows are sequence b's; max_len: an upper bound of a sequence's tokens."""
    cu_tokens: torch.Tensor
    n_tokens: int
    max_len: int

    def struct(self, seqs: Seqs, q_stride: int = 0, k_stride: int = 0, v_stride: int = 0) -> kvg_packed:
        cu = self.cu_tokens
        if not (cu.dtype is torch.int32 and cu.is_contiguous() and cu.numel() == seqs.block_tables.shape[0] + 1):
            raise ValueError("cu_tokens: int32 [batch + 1], contiguous")
        return kvg_packed(self.n_tokens, self.max_len, cu.data_ptr(), q_stride, k_stride, v_stride)


def _token_stride(t: torch.Tensor, n_layers: int, n_tokens: int, heads: int, head_dim: int, dtype: torch.dtype) -> int:
    """Token stride of packed rows [n_layers][n_tokens][heads][head_dim], which may be a view into wider rows."""
    if t.dtype is not dtype or t.shape != (n_layers, n_tokens, heads, head_dim):
        raise ValueError(f"packed rows: {dtype} [{n_layers}][{n_tokens}][{heads}][{head_dim}], got {t.dtype} {tuple(t.shape)}")
    sl, st, sh, sd = t.stride()
    if n_tokens <= 1:                      # a token's rows are n_tokens strides from the next layer's
        st = sl if n_layers > 1 and n_tokens else heads * head_dim
    if (sd != 1 or sh != head_dim and heads > 1 or st < heads * head_dim or
            n_layers > 1 and n_tokens and sl != n_tokens * st):
        raise ValueError("packed rows: heads dense, layers n_tokens rows apart")
    return st


def _on_current_device(*tensors):
    """The packed calls run on the current device's current stream: tensors of another device are refused."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor on {t.device}, the current device is {here}")


def kvg_rotary_frequencies(rt: kvg_rotary, head_dim: int) -> list[float]:
    theta = (ctypes.c_double * 128)()
    _check(_lib.kvg_rotary_frequencies(ctypes.byref(rt), head_dim, theta), "kvg_rotary_frequencies")
    return list(theta[: (rt.rotary_dim or head_dim) // 2])


def kvg_artifact_header_init_rotary(cache: Cache, n_tokens: int, own_pos: int, rt: kvg_rotary) -> kvg_artifact_hdr:
    hdr = kvg_artifact_hdr()
    _check(_lib.kvg_artifact_header_init_rotary(ctypes.byref(cache.struct()), n_tokens, own_pos, ctypes.byref(rt),
                                                ctypes.byref(hdr)), "kvg_artifact_header_init_rotary")
    return hdr


_AXES = struct.Struct("@P8i")       # kvg_axes


@dataclasses.dataclass
class Axes:
    """Positions with several axes: int64 [n_axes][n_tokens] (device); pairs of a head's rotated components for each axis,
    in contiguous sections or in turn (kvg.h)."""
    positions: torch.Tensor
    pairs: tuple
    order: int = KVG_AXES_SECTIONS
    own_frequencies: bool = False

    def struct(self, n_tokens: int) -> kvg_axes:
        pos, n = self.positions, len(self.pairs)
        if not 1 <= n <= KVG_MAX_AXES:
            raise ValueError(f"pairs: of 1 to {KVG_MAX_AXES} axes")
        if not (pos.dtype is torch.int64 and pos.is_contiguous() and pos.shape == (n, n_tokens)):
            raise ValueError("positions: int64 [n_axes][n_tokens], contiguous")
        # packed in one step: a ctypes array and nine fields took half of a small call's marshalling
        return kvg_axes.from_buffer_copy(_AXES.pack(pos.data_ptr(), n, self.order, int(self.own_frequencies), 0, *self.pairs,
                                                    *(0,) * (KVG_MAX_AXES - n)))


def kvg_artifact_header_init_axes(cache: Cache, n_tokens: int, own_pos: int, rt: kvg_rotary, axes: Axes) -> kvg_artifact_hdr:
    """Header of a block of n_tokens tokens at positions with several axes (which it does not read: those of any call do)."""
    hdr = kvg_artifact_hdr()
    _check(_lib.kvg_artifact_header_init_axes(ctypes.byref(cache.struct()), n_tokens, own_pos, ctypes.byref(rt),
                                              ctypes.byref(axes.struct(axes.positions.shape[-1])), ctypes.byref(hdr)),
           "kvg_artifact_header_init_axes")
    return hdr


def _rotate_strides(where: str, x: torch.Tensor, y: torch.Tensor):
    """Token strides of x and y, [n_tokens][n_heads][head_dim] with dense heads."""
    shape, dtype = x.shape, x.dtype
    T, H, D = shape
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise KvgError(-3, where)
    sx, hx, dx = x.stride()
    sy, hy, dy = y.stride()
    if y.dtype is not dtype or y.shape != shape or dx != 1 or dy != 1 or H > 1 and (hx != D or hy != D):
        raise ValueError(f"{where}: x and y alike, heads dense")
    if T <= 1:
        return 0, 0
    if sx < H * D or sy < H * D:           # a broadcast row among them: 0 is the library's word for dense rows
        raise ValueError(f"{where}: a token's rows overlap the next one's")
    return sx, sy


def kvg_rotate(rt: kvg_rotary, positions: torch.Tensor, x: torch.Tensor, y: torch.Tensor, stream=None):
    """y[t][h] = x[t][h] rotated at positions[t] (int64); x, y: [n_tokens][n_heads][head_dim], fp32 or bf16, heads
    dense, any token stride; y may be x."""
    T, H, D = x.shape
    sx, sy = _rotate_strides("kvg_rotate", x, y)
    if not (positions.dtype is torch.int64 and positions.is_contiguous() and positions.numel() == T):
        raise ValueError("positions: int64 [n_tokens], contiguous")
    _on_current_device(positions, x, y)
    _check(_lib.kvg_rotate(ctypes.byref(rt), 1 if x.dtype is torch.bfloat16 else 0, D, T, H, positions.data_ptr(), x.data_ptr(), sx,
                           y.data_ptr(), sy, _stream(stream)), "kvg_rotate")


def kvg_rotate_axes(rt: kvg_rotary, axes: Axes, x: torch.Tensor, y: torch.Tensor, stream=None):
    """kvg_rotate at positions with several axes."""
    T, H, D = x.shape
    sx, sy = _rotate_strides("kvg_rotate_axes", x, y)
    _on_current_device(axes.positions, x, y)
    _check(_lib.kvg_rotate_axes(ctypes.byref(rt), ctypes.byref(axes.struct(T)), 1 if x.dtype is torch.bfloat16 else 0, D, T, H,
                                x.data_ptr(), sx, y.data_ptr(), sy, _stream(stream)), "kvg_rotate_axes")


def _append_args(cache, raw, seqs: Seqs, packed: Packed, norm: HeadNorm | None, n_layers: int, q_raw, k_raw, v_raw, q_out,
                 *others):
    """Checked structs of the calls that append packed tokens: sequences, packed rows, norm."""
    T, D, Hkv = packed.n_tokens, cache.head_dim, cache.n_kv_heads
    sq = 0
    if q_raw is not None:
        sq = _token_stride(q_raw, n_layers, T, cache.n_q_heads, D, raw)
    if q_out is not None:
        if not (q_out.shape == (n_layers, T, cache.n_q_heads, D) and q_out.dtype is raw and q_out.is_contiguous()):
            raise ValueError("q_out: [n_layers][n_tokens][n_q_heads][head_dim] of the raw dtype, contiguous")
    sk, sv = (_token_stride(t, n_layers, T, Hkv, D, raw) for t in (k_raw, v_raw))
    ns = None if norm is None else norm.struct(cache, n_layers)
    _on_current_device(cache.k_pool, cache.v_pool, packed.cu_tokens, seqs.block_tables, seqs.ctx_lens, seqs.start_pos, k_raw,
                       v_raw, q_raw, q_out, *(() if norm is None else (norm.q_weight, norm.k_weight)), *others)
    return (ctypes.byref(seqs.struct()), ctypes.byref(packed.struct(seqs, sq, sk, sv)), None if ns is None else ctypes.byref(ns))


def kvg_norm_append(cache: Cache, seqs: Seqs, packed: Packed, rt: kvg_rotary, norm: HeadNorm | None, layer0: int,
                    n_layers: int, q_raw: torch.Tensor | None, k_raw: torch.Tensor, v_raw: torch.Tensor,
                    q_out: torch.Tensor | None, stream=None):
    """Norm, rotation and append of packed tokens.  q_raw, k_raw, v_raw: [n_layers][n_tokens][heads][head_dim] of the raw
    dtype, views into wider rows allowed; q_out: dense (q_raw and q_out: both None for keys and values alone)."""
    s, p, ns = _append_args(cache, cache.raw_dtype, seqs, packed, norm, n_layers, q_raw, k_raw, v_raw, q_out)
    _check(_lib.kvg_norm_append(ctypes.byref(cache.struct()), s, p, ctypes.byref(rt), ns, layer0, n_layers, _ptr(q_raw),
                                _ptr(k_raw), _ptr(v_raw), _ptr(q_out), _stream(stream)), "kvg_norm_append")


def kvg_norm_append_axes(cache: Cache, seqs: Seqs, packed: Packed, rt: kvg_rotary, axes: Axes, norm: HeadNorm | None,
                         layer0: int, n_layers: int, q_raw: torch.Tensor | None, k_raw: torch.Tensor, v_raw: torch.Tensor,
                         q_out: torch.Tensor | None, stream=None):
    """kvg_norm_append at positions with several axes (seqs.start_pos is not read)."""
    s, p, ns = _append_args(cache, cache.raw_dtype, seqs, packed, norm, n_layers, q_raw, k_raw, v_raw, q_out, axes.positions)
    _check(_lib.kvg_norm_append_axes(ctypes.byref(cache.struct()), s, p, ctypes.byref(rt),
                                     ctypes.byref(axes.struct(packed.n_tokens)), ns, layer0, n_layers, _ptr(q_raw), _ptr(k_raw),
                                     _ptr(v_raw), _ptr(q_out), _stream(stream)), "kvg_norm_append_axes")


def kvg_packed_attn_workspace_bytes(cache: Cache, seqs: Seqs, packed: Packed, n_layers: int) -> int:
    return _lib.kvg_packed_attn_workspace_bytes(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()),
                                                ctypes.byref(packed.struct(seqs)), n_layers)


def packed_attn_workspace(cache: Cache, seqs: Seqs, packed: Packed, n_layers: int) -> torch.Tensor:
    """Scratch for kvg_packed_attn calls of this batch's bounds."""
    return torch.empty(max(kvg_packed_attn_workspace_bytes(cache, seqs, packed, n_layers), 256), dtype=torch.uint8,
                       device=cache.k_pool.device)


def kvg_packed_attn(cache: Cache, seqs: Seqs, packed: Packed, layer0: int, n_layers: int, q: torch.Tensor, scale: float,
                    out: torch.Tensor, ws: torch.Tensor, stream=None):
    """Causal attention of packed tokens over the cache.  q: [n_layers][n_tokens][n_q_heads][head_dim] of the raw dtype,
    rotated, any token stride; out: the same, dense."""
    raw, T, D, Hq = cache.raw_dtype, packed.n_tokens, cache.head_dim, cache.n_q_heads
    sq = _token_stride(q, n_layers, T, Hq, D, raw)
    if not (out.shape == (n_layers, T, Hq, D) and out.dtype is raw and out.is_contiguous()):
        raise ValueError("out: [n_layers][n_tokens][n_q_heads][head_dim] of the raw dtype, contiguous")
    if not ws.is_contiguous():
        raise ValueError("ws: contiguous")
    _on_current_device(cache.k_pool, cache.v_pool, packed.cu_tokens, seqs.block_tables, seqs.ctx_lens, q, out, ws)
    _check(_lib.kvg_packed_attn(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()),
                                ctypes.byref(packed.struct(seqs, sq)), layer0, n_layers, _ptr(q), scale, _ptr(out),
                                _ptr(ws), ws.nbytes, _stream(stream)), "kvg_packed_attn")


@dataclasses.dataclass
class Int8Cache:
    """Paged pools of 8-bit integers [n_layers][n_pages][n_kv_heads][page_size][head_dim] (torch.int8) and the scale of every page and
    KV head, fp32 [n_layers][n_pages][n_kv_heads]: a value is its integer times its scale."""
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor
    n_q_heads: int
    windows: tuple | None = None       # per-layer sliding window (0 = full causal), or None

    @staticmethod
    def allocate(n_layers, n_pages, n_q_heads, n_kv_heads, head_dim, device="cuda", page_size=16, windows=None):
        pages = Cache.allocate(n_layers, n_pages, n_q_heads, n_kv_heads, head_dim, torch.int8, device, page_size, windows)
        scales = [torch.empty((n_layers, n_pages, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2)]
        return Int8Cache(pages.k_pool, pages.v_pool, *scales, n_q_heads, pages.windows)

    @property
    def n_layers(self):
        return self.k_pool.shape[0]

    @property
    def n_pages(self):
        return self.k_pool.shape[1]

    @property
    def n_kv_heads(self):
        return self.k_pool.shape[2]

    @property
    def page_size(self):
        return self.k_pool.shape[3]

    @property
    def head_dim(self):
        return self.k_pool.shape[4]

    @property
    def raw_dtype(self) -> torch.dtype:
        return torch.bfloat16

    def struct(self) -> kvg_int8_cache:
        k, v, ks, vs = self.k_pool, self.v_pool, self.k_scale, self.v_scale
        if k.dtype is not torch.int8:
            raise ValueError("pools: torch.int8")
        shape = k.shape[:3]
        if not (ks.dtype is vs.dtype is torch.float32 and ks.shape == vs.shape == shape and ks.is_contiguous() and
                vs.is_contiguous()):
            raise ValueError("scales: fp32 [n_layers][n_pages][n_kv_heads], contiguous")
        pages = _pages_struct(k, v, self.n_q_heads, KVG_INT8, self.windows)
        c = kvg_int8_cache(pages, ks.data_ptr(), vs.data_ptr())
        c._windows_keepalive = getattr(pages, "_windows_keepalive", None)     # the copy holds the raw pointer too
        return c

    def tensors(self):
        return self.k_pool, self.v_pool, self.k_scale, self.v_scale


def kvg_int8_append(cache: Int8Cache, seqs: Seqs, packed: Packed, rt: kvg_rotary, norm: HeadNorm | None, layer0: int,
                    n_layers: int, q_raw: torch.Tensor | None, k_raw: torch.Tensor, v_raw: torch.Tensor,
                    q_out: torch.Tensor | None, axes: Axes | None = None, stream=None):
    """Norm, rotation and append of packed tokens to an int8 cache; rows as kvg_norm_append's, bf16.  axes: positions with
    several axes in the place of seqs.start_pos + index."""
    s, p, ns = _append_args(cache, torch.bfloat16, seqs, packed, norm, n_layers, q_raw, k_raw, v_raw, q_out, cache.k_scale,
                            cache.v_scale, None if axes is None else axes.positions)
    _check(_lib.kvg_int8_append(ctypes.byref(cache.struct()), s, p, ctypes.byref(rt),
                                None if axes is None else ctypes.byref(axes.struct(packed.n_tokens)), ns, layer0, n_layers,
                                _ptr(q_raw), _ptr(k_raw), _ptr(v_raw), _ptr(q_out), _stream(stream)), "kvg_int8_append")


def kvg_int8_attn_workspace_bytes(cache: Int8Cache, seqs: Seqs, packed: Packed, n_layers: int) -> int:
    return _lib.kvg_int8_attn_workspace_bytes(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()),
                                              ctypes.byref(packed.struct(seqs)), n_layers)


def int8_attn_workspace(cache: Int8Cache, seqs: Seqs, packed: Packed, n_layers: int) -> torch.Tensor:
    """Scratch for kvg_int8_attn calls of this batch's bounds."""
    return torch.empty(max(kvg_int8_attn_workspace_bytes(cache, seqs, packed, n_layers), 256), dtype=torch.uint8,
                       device=cache.k_pool.device)


def kvg_int8_attn(cache: Int8Cache, seqs: Seqs, packed: Packed, layer0: int, n_layers: int, q: torch.Tensor, scale: float,
                  out: torch.Tensor, ws: torch.Tensor, stream=None):
    """kvg_packed_attn over an int8 cache.  q: bf16 [n_layers][n_tokens][n_q_heads][head_dim], rotated, any token stride;
    out: the same, dense."""
    T, D, Hq = packed.n_tokens, cache.head_dim, cache.n_q_heads
    sq = _token_stride(q, n_layers, T, Hq, D, torch.bfloat16)
    if not (out.shape == (n_layers, T, Hq, D) and out.dtype is torch.bfloat16 and out.is_contiguous()):
        raise ValueError("out: bf16 [n_layers][n_tokens][n_q_heads][head_dim], contiguous")
    if not ws.is_contiguous():
        raise ValueError("ws: contiguous")
    _on_current_device(*cache.tensors(), packed.cu_tokens, seqs.block_tables, seqs.ctx_lens, q, out, ws)
    _check(_lib.kvg_int8_attn(ctypes.byref(cache.struct()), ctypes.byref(seqs.struct()), ctypes.byref(packed.struct(seqs, sq)),
                              layer0, n_layers, _ptr(q), scale, _ptr(out), _ptr(ws), ws.nbytes, _stream(stream)),
           "kvg_int8_attn")


def kvg_int8_payload_bytes(cache: Int8Cache, n_tokens: int) -> int:
    return _lib.kvg_int8_payload_bytes(ctypes.byref(cache.struct()), n_tokens)


def kvg_int8_header_init(cache: Int8Cache, n_tokens: int, own_pos: int) -> kvg_artifact_hdr:
    hdr = kvg_artifact_hdr()
    _check(_lib.kvg_int8_header_init(ctypes.byref(cache.struct()), n_tokens, own_pos, ctypes.byref(hdr)), "kvg_int8_header_init")
    return hdr


def _block_table(row: torch.Tensor):
    if not (row.dtype is torch.int32 and row.is_contiguous()):
        raise ValueError("block table: int32, contiguous")


def kvg_int8_deposit(cache: Int8Cache, block_table_row: torch.Tensor, first_token: int, n_tokens: int, payload: torch.Tensor,
                     stream=None):
    """kvg_deposit of an int8 block: its integers, then its scales."""
    _block_table(block_table_row)
    on_device = _payload_ok(payload, kvg_int8_payload_bytes(cache, n_tokens), "kvg_int8_payload_bytes(cache, n_tokens) bytes")
    _on_current_device(*cache.tensors(), block_table_row, on_device)
    _check(_lib.kvg_int8_deposit(ctypes.byref(cache.struct()), _ptr(block_table_row), block_table_row.numel(), first_token,
                                 n_tokens, _ptr(payload), _stream(stream)), "kvg_int8_deposit")


def kvg_int8_graft(cache: Int8Cache, hdr: kvg_artifact_hdr, payload, block_table_row: torch.Tensor, first_token: int,
                   target_pos: int, stream=None):
    """kvg_graft of an int8 block, at its own position."""
    _block_table(block_table_row)
    on_device = _payload_ok(payload, hdr.payload_bytes, "the header's payload_bytes")
    _on_current_device(*cache.tensors(), block_table_row, on_device)
    _check(_lib.kvg_int8_graft(ctypes.byref(cache.struct()), ctypes.byref(hdr), _payload_ptr(payload), _ptr(block_table_row),
                               block_table_row.numel(), first_token, target_pos, _stream(stream)), "kvg_int8_graft")


def kvg_leaf_digests(data: torch.Tensor, leaf_bytes: int, digests: torch.Tensor, n_bytes: int | None = None,
                     stream=None):
    """SHA-256 of each leaf of `data`'s bytes into `digests` (uint8 [n_leaves][32], device)."""
    nb = data.nbytes if n_bytes is None else n_bytes
    _check(_lib.kvg_leaf_digests(_ptr(data), nb, leaf_bytes, _ptr(digests), _stream(stream)), "kvg_leaf_digests")


def kvg_merkle_workspace_bytes(n_leaves: int) -> int:
    return _lib.kvg_merkle_workspace_bytes(n_leaves)


def kvg_merkle_root(digests: torch.Tensor, n_leaves: int, root: torch.Tensor, ws: torch.Tensor, stream=None):
    _check(_lib.kvg_merkle_root(_ptr(digests), n_leaves, _ptr(root), _ptr(ws), ws.nbytes, _stream(stream)),
           "kvg_merkle_root")


def kvg_dedup_workspace_bytes(n_leaves: int) -> int:
    return _lib.kvg_dedup_workspace_bytes(n_leaves)


def kvg_dedup_map(digests: torch.Tensor, n_leaves: int, first_index: torch.Tensor, n_unresolved: torch.Tensor,
                  ws: torch.Tensor, stream=None):
    _check(_lib.kvg_dedup_map(_ptr(digests), n_leaves, _ptr(first_index), _ptr(n_unresolved), _ptr(ws), ws.nbytes,
                              _stream(stream)), "kvg_dedup_map")


def kvg_logits_packed_bytes(vocab: int, hidden: int) -> int:
    return _lib.kvg_logits_packed_bytes(vocab, hidden)


def kvg_logits_pack(w: torch.Tensor, packed: torch.Tensor, stream=None):
    """w: bf16 [V][H] row-major; packed: kvg_logits_packed_bytes(V, H) bytes (device)."""
    V, H = w.shape
    if not (w.dtype == torch.bfloat16 and w.is_contiguous() and packed.nbytes >= kvg_logits_packed_bytes(V, H)):
        raise ValueError("w: bf16, contiguous; packed: kvg_logits_packed_bytes(V, H) bytes")
    _check(_lib.kvg_logits_pack(_ptr(w), V, H, _ptr(packed), _stream(stream)), "kvg_logits_pack")


def kvg_logits_workspace_bytes(rows: int, hidden: int) -> int:
    return _lib.kvg_logits_workspace_bytes(rows, hidden)


def kvg_logits(hidden: torch.Tensor, w_packed: torch.Tensor, vocab: int, cap: float, out: torch.Tensor,
               ws: torch.Tensor, stream=None):
    """hidden: fp32 [rows][H]; w_packed: as kvg_logits_pack left it; out: fp32 [rows][vocab]."""
    rows, H = hidden.shape
    if not (tuple(out.shape) == (rows, vocab) and w_packed.nbytes >= kvg_logits_packed_bytes(vocab, H) and
            hidden.dtype == torch.float32 and out.dtype == torch.float32 and
            hidden.is_contiguous() and w_packed.is_contiguous() and out.is_contiguous()):
        raise ValueError("hidden: fp32 [rows][H]; w_packed: kvg_logits_packed_bytes(vocab, H) bytes; out: fp32 [rows][vocab]; contiguous")
    _check(_lib.kvg_logits(_ptr(hidden), rows, H, _ptr(w_packed), vocab, cap, _ptr(out), _ptr(ws), ws.nbytes,
                           _stream(stream)), "kvg_logits")


def kvg_logit_compare(a: torch.Tensor, b: torch.Tensor, kl: torch.Tensor, argmax_a: torch.Tensor,
                      argmax_b: torch.Tensor, stream=None):
    """a, b: fp32 [rows][V]; kl: fp64 [rows]; argmax_a, argmax_b: int32 [rows] (all device)."""
    rows, V = a.shape
    if not (tuple(b.shape) == (rows, V) and a.dtype == b.dtype == torch.float32 and a.is_contiguous() and b.is_contiguous()):
        raise ValueError("a, b: fp32 [rows][V], contiguous")
    if not (kl.dtype == torch.float64 and argmax_a.dtype == argmax_b.dtype == torch.int32 and
            kl.numel() >= rows and argmax_a.numel() >= rows and argmax_b.numel() >= rows):
        raise ValueError("kl: fp64 [rows]; argmax_a, argmax_b: int32 [rows]")
    _check(_lib.kvg_logit_compare(_ptr(a), _ptr(b), rows, V, _ptr(kl), _ptr(argmax_a), _ptr(argmax_b),
                                  _stream(stream)), "kvg_logit_compare")


def kvg_sample_workspace_bytes(rows: int, vocab: int) -> int:
    return _lib.kvg_sample_workspace_bytes(rows, vocab)


def sample_workspace(rows: int, vocab: int, device="cuda") -> torch.Tensor:
    """Scratch for kvg_sample calls of these sizes."""
    return torch.empty(max(kvg_sample_workspace_bytes(rows, vocab), 256), dtype=torch.uint8, device=device)


def kvg_sample(logits: torch.Tensor, temperature: torch.Tensor, uniform: torch.Tensor, tokens: torch.Tensor, ws: torch.Tensor,
               top_k: torch.Tensor | None = None, top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None,
               logprobs: torch.Tensor | None = None, stream=None):
    """tokens (int32 [rows]) sampled from logits (fp32 [rows][vocab], any row stride) with one random number a row (uniform: fp64 [rows]);
    temperature, top_p, min_p: fp32 [rows], top_k: int32 [rows] (None: no such limit); logprobs: fp32 [rows] or None."""
    rows, V = logits.shape
    if logits.dtype is not torch.float32 or V > 1 and logits.stride(1) != 1:
        raise ValueError("logits: fp32 [rows][vocab], rows dense")
    stride = logits.stride(0) if rows > 1 else V
    if stride < V:                         # a broadcast row among them: 0 is the library's word for dense rows
        raise ValueError("logits: a row overlaps the next one")
    for name, t, dtype in (("temperature", temperature, torch.float32), ("uniform", uniform, torch.float64),
                           ("tokens", tokens, torch.int32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                           ("min_p", min_p, torch.float32), ("logprobs", logprobs, torch.float32)):
        if t is not None and not (t.dtype is dtype and t.shape == (rows,) and t.is_contiguous()):
            raise ValueError(f"{name}: {dtype} [rows], contiguous")
    if not ws.is_contiguous():
        raise ValueError("ws: contiguous")
    _on_current_device(logits, temperature, uniform, tokens, ws, top_k, top_p, min_p, logprobs)
    s = kvg_sampling(_ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p))
    _check(_lib.kvg_sample(_ptr(logits), stride, rows, V, ctypes.byref(s), _ptr(uniform), _ptr(tokens), _ptr(logprobs), _ptr(ws),
                           ws.nbytes, _stream(stream)), "kvg_sample")


def raw_call(name: str, *args):
    """Direct call of an exported symbol with pre-marshalled ctypes arguments (for validation tests)."""
    return getattr(_lib, name)(*args)
