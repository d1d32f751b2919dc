"""ctypes binding of the key-value cache operators (see include/fastrack_kv.h for the contract).

Argument marshalling only, like :mod:`paper_2410_15240_b200.fastrack`: buffers are integer device addresses
(``tensor.data_ptr()``), streams the integer ``cudaStream_t``.  The structs are ctypes structures with the header's field
names; they may be kept and passed to many calls.  Results other than OK raise :class:`fastrack.FastrackError`.
"""
from __future__ import annotations

import ctypes

from .fastrack import OK, FastrackError, _lib

BF16, F16 = 0, 1
INT8, E4M3 = 0, 1
ROTARY_NONE, ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1, 2
FREQ_PLAIN, FREQ_LINEAR, FREQ_BASE, FREQ_RAMP = 0, 1, 2, 3

EXPORTS = ("fastrack_kv_create", "fastrack_kv_destroy", "fastrack_kv_page_bytes", "fastrack_kv_tail_bytes", "fastrack_kv_last_cuda_error",
           "fastrack_kv_launch_count", "fastrack_rotary_frequencies", "fastrack_rotary", "fastrack_kv_append", "fastrack_kv_read",
           "fastrack_kv_attention_workspace", "fastrack_kv_attention", "fastrack_kv_evict")

_vp, _sz, _int, _i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64


class Config(ctypes.Structure):
    _fields_ = [("dtype", _int), ("format", _int), ("q_heads", _int), ("kv_heads", _int), ("head_dim", _int), ("block_tokens", _int),
                ("rotary", _int), ("rotary_dim", _int), ("frequencies", ctypes.POINTER(ctypes.c_double)), ("rotary_gain", ctypes.c_float),
                ("softmax_scale", ctypes.c_float)]


class Batch(ctypes.Structure):
    """The sequences of a call: fastrack_kv_batch."""
    _fields_ = [("n_seqs", _int), ("total_new", _int), ("max_new", _int), ("max_len", _int), ("pool_pages", _int), ("table_stride", _int),
                ("d_pool", _vp), ("d_tail", _vp), ("d_table", _vp), ("d_lens", _vp), ("d_starts", _vp), ("d_positions", _vp)]


class Rows(ctypes.Structure):
    """16-bit vectors of (token, head): fastrack_kv_rows.  Strides in values."""
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class Eviction(ctypes.Structure):
    """One call's eviction: fastrack_kv_eviction."""
    _fields_ = [("n_seqs", _int), ("table_stride", _int), ("mass_stride", _int), ("budget", _int), ("keep_first", _int), ("keep_last", _int),
                ("d_table", _vp), ("d_lens", _vp), ("d_mass", _vp), ("d_table_out", _vp), ("d_lens_out", _vp), ("d_mass_out", _vp),
                ("d_evicted", _vp), ("d_n_evicted", _vp)]


_batch_p, _rows_p = ctypes.POINTER(Batch), ctypes.POINTER(Rows)
_lib.fastrack_kv_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(_vp)]
_lib.fastrack_kv_destroy.restype = None
_lib.fastrack_kv_destroy.argtypes = [_vp]
for _name in ("fastrack_kv_page_bytes", "fastrack_kv_tail_bytes"):
    getattr(_lib, _name).restype = _sz
    getattr(_lib, _name).argtypes = [_vp]
_lib.fastrack_kv_last_cuda_error.argtypes = [_vp]
_lib.fastrack_kv_launch_count.restype = ctypes.c_uint64
_lib.fastrack_kv_launch_count.argtypes = [_vp]
_lib.fastrack_rotary_frequencies.argtypes = [_int, ctypes.c_double, _int, ctypes.c_double, ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                             ctypes.POINTER(ctypes.c_float)]
_lib.fastrack_rotary.argtypes = [_vp, _i64, _int, _rows_p, _rows_p, _vp, _int, _vp]
_lib.fastrack_kv_append.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _rows_p, _rows_p, _vp]
_lib.fastrack_kv_read.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _vp]
_lib.fastrack_kv_attention_workspace.restype = _sz
_lib.fastrack_kv_attention_workspace.argtypes = [_vp, _batch_p, _int]
_lib.fastrack_kv_attention.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _vp, _int, _vp, _vp, _int, _vp, _sz, _vp]
_lib.fastrack_kv_evict.argtypes = [_vp, ctypes.POINTER(Eviction), _vp]


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: int = FREQ_PLAIN, factor: float = 1.0, original_len: float = 0.0):
    """-> (list of radians per position, gain) for KvCache(frequencies=..., rotary_gain=...)."""
    out, gain = (ctypes.c_double * max(1, rotary_dim // 2))(), ctypes.c_float()
    rc = _lib.fastrack_rotary_frequencies(rotary_dim, base, scaling, factor, original_len, out, ctypes.byref(gain))
    if rc != OK:
        raise FastrackError(rc)
    return list(out), gain.value


class KvCache:
    """One shape of cache on the current device (RAII over fastrack_kv_create / _destroy)."""

    def __init__(self, dtype: int, format: int, q_heads: int, kv_heads: int, head_dim: int, block_tokens: int, rotary: int = ROTARY_NONE,
                 frequencies=None, rotary_gain: float = 1.0, softmax_scale: float = 0.0):
        self.handle = None
        frequencies = [] if frequencies is None else [float(f) for f in frequencies]     # any sequence, arrays and tensors among them
        table = (ctypes.c_double * max(1, len(frequencies)))(*frequencies)
        config = Config(dtype, format, q_heads, kv_heads, head_dim, block_tokens, rotary, 2 * len(frequencies), table, rotary_gain, softmax_scale)
        handle = _vp()
        rc = _lib.fastrack_kv_create(ctypes.byref(config), ctypes.byref(handle))
        if rc != OK:
            raise FastrackError(rc)
        self.handle = handle
        self.page_bytes = int(_lib.fastrack_kv_page_bytes(handle))
        self.tail_bytes = int(_lib.fastrack_kv_tail_bytes(handle))

    def _check(self, rc: int) -> None:
        if rc != OK:
            raise FastrackError(rc, _lib.fastrack_kv_last_cuda_error(self.handle))

    def rotary(self, tokens: int, heads: int, x: Rows, out: Rows, d_positions: int, inverse=False, stream: int = 0) -> None:
        self._check(_lib.fastrack_rotary(self.handle, tokens, heads, x, out, d_positions, inverse, stream))

    def append(self, batch: Batch, k: Rows, v: Rows, q: Rows = None, q_out: Rows = None, stream: int = 0) -> None:
        self._check(_lib.fastrack_kv_append(self.handle, batch, k, v, q, q_out, stream))

    def read(self, batch: Batch, k_out: Rows, v_out: Rows, stream: int = 0) -> None:
        self._check(_lib.fastrack_kv_read(self.handle, batch, k_out, v_out, stream))

    def workspace_bytes(self, batch: Batch, with_mass: bool) -> int:
        return int(_lib.fastrack_kv_attention_workspace(self.handle, batch, with_mass))

    def attention(self, batch: Batch, q: Rows, out: Rows, d_workspace: int, workspace_bytes: int, d_lse: int = 0, window: int = 0,
                  d_mass_in: int = 0, d_mass_out: int = 0, mass_stride: int = 0, stream: int = 0) -> None:
        self._check(_lib.fastrack_kv_attention(self.handle, batch, q, out, d_lse, window, d_mass_in, d_mass_out, mass_stride, d_workspace,
                                               workspace_bytes, stream))

    def evict(self, eviction: Eviction, stream: int = 0) -> None:
        self._check(_lib.fastrack_kv_evict(self.handle, eviction, stream))

    @property
    def launches(self) -> int:
        return int(_lib.fastrack_kv_launch_count(self.handle))

    def close(self) -> None:
        if self.handle is not None:
            _lib.fastrack_kv_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
