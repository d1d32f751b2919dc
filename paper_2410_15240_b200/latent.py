"""ctypes binding of the latent cache operators (see include/fastrack_latent.h for the contract).

Argument marshalling only, like :mod:`paper_2410_15240_b200.kv`, whose constants and :class:`kv.Rows` it shares: buffers are integer device
addresses (``tensor.data_ptr()``), streams the integer ``cudaStream_t``.  Results other than OK raise :class:`fastrack.FastrackError`.
"""
from __future__ import annotations

import ctypes

from .fastrack import OK, FastrackError, _lib
from .kv import ROTARY_NONE, Rows, _rows_p

TREE_MOST = 1024                        # new tokens of a sequence, where they are a tree

EXPORTS = ("fastrack_latent_create", "fastrack_latent_destroy", "fastrack_latent_page_bytes", "fastrack_latent_last_cuda_error",
           "fastrack_latent_launch_count", "fastrack_latent_append", "fastrack_latent_attention_workspace", "fastrack_latent_attention",
           "fastrack_latent_expand", "fastrack_latent_prompt_workspace", "fastrack_latent_prompt", "fastrack_latent_accept")

_vp, _sz, _int, _i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64


class Config(ctypes.Structure):
    _fields_ = [("dtype", _int), ("heads", _int), ("latent_dim", _int), ("rope_dim", _int), ("key_dim", _int), ("value_dim", _int), ("block_tokens", _int),
                ("rotary", _int), ("frequencies", ctypes.POINTER(ctypes.c_double)), ("rotary_gain", ctypes.c_float), ("norm_eps", ctypes.c_float),
                ("softmax_scale", ctypes.c_float)]


class Batch(ctypes.Structure):
    """The sequences of a call: fastrack_latent_batch."""
    _fields_ = [("n_seqs", _int), ("total_new", _int), ("max_new", _int), ("max_len", _int), ("pool_pages", _int), ("table_stride", _int),
                ("d_pool", _vp), ("d_table", _vp), ("d_lens", _vp), ("d_starts", _vp), ("d_positions", _vp)]


class Acceptance(ctypes.Structure):
    """A drafted tree and what the model chose: fastrack_latent_acceptance."""
    _fields_ = [("d_parents", _vp), ("d_tokens", _vp), ("d_choices", _vp), ("d_path", _vp), ("d_n_accepted", _vp), ("d_next", _vp), ("d_lens_out", _vp)]


_batch_p = ctypes.POINTER(Batch)
_lib.fastrack_latent_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(_vp)]
_lib.fastrack_latent_destroy.restype = None
_lib.fastrack_latent_destroy.argtypes = [_vp]
_lib.fastrack_latent_page_bytes.restype = _sz
_lib.fastrack_latent_page_bytes.argtypes = [_vp]
_lib.fastrack_latent_last_cuda_error.argtypes = [_vp]
_lib.fastrack_latent_launch_count.restype = ctypes.c_uint64
_lib.fastrack_latent_launch_count.argtypes = [_vp]
_lib.fastrack_latent_append.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _vp, _rows_p, _rows_p, _vp]
for _name in ("fastrack_latent_attention_workspace", "fastrack_latent_prompt_workspace"):
    getattr(_lib, _name).restype = _sz
    getattr(_lib, _name).argtypes = [_vp, _batch_p]
_lib.fastrack_latent_attention.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _rows_p, _vp, _vp, _vp, _sz, _vp]
_lib.fastrack_latent_expand.argtypes = [_vp, _batch_p, _vp, _rows_p, _rows_p, _vp, _int, _vp]
_lib.fastrack_latent_prompt.argtypes = [_vp, _batch_p, _rows_p, _rows_p, _rows_p, _rows_p, _vp, _int, _rows_p, _vp, _vp, _sz, _vp]
_lib.fastrack_latent_accept.argtypes = [_vp, _batch_p, ctypes.POINTER(Acceptance), _vp]


class LatentCache:
    """One shape of latent cache on the current device (RAII over fastrack_latent_create / _destroy)."""

    def __init__(self, dtype: int, heads: int, latent_dim: int, rope_dim: int, key_dim: int, value_dim: int, block_tokens: int, rotary: int = ROTARY_NONE,
                 frequencies=None, rotary_gain: float = 1.0, norm_eps: float = 1e-6, softmax_scale: float = 0.0):
        self.handle = None
        table = None
        if frequencies is not None:                                       # any sequence, arrays and tensors among them
            values = [float(f) for f in frequencies]
            if len(values) != rope_dim // 2:
                raise ValueError(f"{rope_dim // 2} frequencies wanted, {len(values)} given")
            table = (ctypes.c_double * max(1, len(values)))(*values)
        config = Config(dtype, heads, latent_dim, rope_dim, key_dim, value_dim, block_tokens, rotary, table, rotary_gain, norm_eps, softmax_scale)
        handle = _vp()
        rc = _lib.fastrack_latent_create(ctypes.byref(config), ctypes.byref(handle))
        if rc != OK:
            raise FastrackError(rc)
        self.handle = handle
        self.page_bytes = int(_lib.fastrack_latent_page_bytes(handle))

    def _check(self, rc: int) -> None:
        if rc != OK:
            raise FastrackError(rc, _lib.fastrack_latent_last_cuda_error(self.handle))

    def append(self, batch: Batch, latents: Rows, key: Rows, d_norm_weight: int = 0, q: Rows = None, q_out: Rows = None, stream: int = 0) -> None:
        self._check(_lib.fastrack_latent_append(self.handle, batch, latents, key, d_norm_weight, q, q_out, stream))

    def workspace_bytes(self, batch: Batch) -> int:
        return int(_lib.fastrack_latent_attention_workspace(self.handle, batch))

    def attention(self, batch: Batch, q: Rows, q_rope: Rows, out: Rows, d_workspace: int, workspace_bytes: int, d_lse: int = 0, d_parents: int = 0,
                  stream: int = 0) -> None:
        self._check(_lib.fastrack_latent_attention(self.handle, batch, q, q_rope, out, d_lse, d_parents, d_workspace, workspace_bytes, stream))

    def expand(self, batch: Batch, d_weights: int, k_out: Rows, v_out: Rows, d_key_starts: int, total_keys: int, stream: int = 0) -> None:
        self._check(_lib.fastrack_latent_expand(self.handle, batch, d_weights, k_out, v_out, d_key_starts, total_keys, stream))

    def prompt_workspace_bytes(self, batch: Batch) -> int:
        return int(_lib.fastrack_latent_prompt_workspace(self.handle, batch))

    def prompt(self, batch: Batch, q: Rows, q_rope: Rows, k: Rows, v: Rows, d_key_starts: int, total_keys: int, out: Rows, d_workspace: int = 0,
               workspace_bytes: int = 0, d_lse: int = 0, stream: int = 0) -> None:
        self._check(_lib.fastrack_latent_prompt(self.handle, batch, q, q_rope, k, v, d_key_starts, total_keys, out, d_lse, d_workspace, workspace_bytes,
                                                stream))

    def accept(self, batch: Batch, acceptance: Acceptance, stream: int = 0) -> None:
        self._check(_lib.fastrack_latent_accept(self.handle, batch, acceptance, stream))

    @property
    def launches(self) -> int:
        return int(_lib.fastrack_latent_launch_count(self.handle))

    def close(self) -> None:
        if self.handle is not None:
            _lib.fastrack_latent_destroy(self.handle)
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
