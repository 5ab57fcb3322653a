"""Thin ctypes binding of the paged key / value cache in 4 bits in libftattn.so: argument marshalling only.

It raises if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import numpy as np

from . import ftattn as _base
from .ftprompt import ints, load_library as _load_prompt, rows

F16, BF16, F32 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4

EXPORTS = ("ftcache_create", "ftcache_get_config", "ftcache_page_bytes", "ftcache_append", "ftcache_read", "ftcache_attend",
           "ftcache_report", "ftcache_destroy", "ftcache_last_error")


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("pages", C.c_int32), ("page_size", C.c_int32), ("in_dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("softmax_scale", C.c_float), ("max_batch", C.c_int32),
                ("device", C.c_int32)]


class ReportView(C.Structure):
    _fields_ = [("refused_tokens", C.c_int64), ("refused_sequences", C.c_int64)]


_typed = False
_uint8 = _int32 = _float32 = None          # torch's, once load_library has run


class FtCacheError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ftcache error {code}: {msg}")
        self.code = code


def load_library() -> C.CDLL:
    """The shared library with the ftcache_* prototypes set; raises if it is not built."""
    global _typed, _uint8, _int32, _float32
    lib = _load_prompt()          # (which knows torch's types)
    if not _typed:
        import torch
        _uint8, _int32, _float32 = torch.uint8, torch.int32, torch.float32
        p = C.c_void_p
        lib.ftcache_create.argtypes = [C.POINTER(Config), C.POINTER(p)]
        lib.ftcache_get_config.argtypes = [p, C.POINTER(Config)]
        lib.ftcache_page_bytes.argtypes = [p]
        lib.ftcache_append.argtypes = [p, p, p, p, C.c_int32, p, p, p, p, p, p]
        lib.ftcache_read.argtypes = [p, p, p, p, p, p]
        lib.ftcache_attend.argtypes = [p, p, C.c_int32, p, p, C.c_int32, C.c_int64, p, p, p]
        lib.ftcache_report.argtypes = [p, C.POINTER(ReportView)]
        lib.ftcache_destroy.argtypes = [p]
        lib.ftcache_last_error.argtypes = [p]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        lib.ftcache_last_error.restype = C.c_char_p
        lib.ftcache_page_bytes.restype = C.c_int64
        _typed = True
    return lib


def rotation_table(positions: int, rotary_dim: int, base: float = 10000.0) -> np.ndarray:
    """float32 [positions, rotary_dim]: cosines, then sines, of position * base^(-2i / rotary_dim), taken in 64 bits (in 32, the angle
    of a far position is off by more than the rotation of neighbours)."""
    speed = base ** (-np.arange(0, rotary_dim, 2, dtype=np.float64) / rotary_dim)
    angle = np.arange(positions, dtype=np.float64)[:, None] * speed
    return np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)


_PLACES = struct.Struct("@iiPPPiq")          # ftcache_places
_NONE = bytes(24)                            # ftcache_rows without a tensor


def _count(t, name: str) -> int:
    try:
        return t.shape[0]
    except (AttributeError, IndexError):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}") from None


class FtCache:
    """One context of the C library: a pool of pages of one geometry on one device.

    The pool itself is the caller's: a contiguous uint8 device tensor of pages * page_bytes elements.  Tables: int32 device tensors,
    page_table [batch, width] (rows may lie apart), lengths and starts [batch], cu_seqlens [batch + 1]."""

    def __init__(self, heads: int, kv_heads: int, head_dim: int, pages: int, page_size: int, in_dtype: int,
                 out_dtype: Optional[int] = None, rotary_dim: int = 0, interleaved: bool = False, softmax_scale: float = 0.0,
                 max_batch: int = 256, device: int = 0):
        self.handle = C.c_void_p()
        self.lib = load_library()
        cfg = Config(C.sizeof(Config), heads, kv_heads, head_dim, pages, page_size, in_dtype, in_dtype if out_dtype is None else out_dtype,
                     rotary_dim, int(bool(interleaved)), softmax_scale, max_batch, device)
        rc = self.lib.ftcache_create(C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            raise FtCacheError(rc, self.lib.ftcache_last_error(None).decode())
        self.config = Config()
        self.lib.ftcache_get_config(self.handle, C.byref(self.config))
        e = self.config
        self.page_bytes = self.lib.ftcache_page_bytes(self.handle)
        self._q = (e.heads, e.head_dim, e.in_dtype, e.device)
        self._kv = (e.kv_heads, e.head_dim, e.in_dtype, e.device)
        self._device, self._bytes, self._rotary = e.device, e.pages * self.page_bytes, e.rotary_dim
        self._o = (e.heads, e.head_dim, e.out_dtype, e.device, True)

    def _check(self, rc: int) -> None:
        if rc != OK:
            raise FtCacheError(rc, self.lib.ftcache_last_error(self.handle).decode())

    def _pool(self, pool) -> int:
        if isinstance(pool, _base._torch_tensor) and pool.dtype is _uint8 and pool.get_device() == self._device and pool.is_contiguous() and pool.numel() == self._bytes:
            return pool.data_ptr()
        if not hasattr(pool, "data_ptr"):
            raise TypeError(f"pool: expected a device tensor, got {type(pool).__name__}")
        if pool.get_device() != self._device:
            raise ValueError(f"pool: tensor is not on device {self._device}")
        raise ValueError(f"pool: expected {self._bytes} contiguous elements of torch.uint8, got {pool.numel()} of {pool.dtype}")

    def _table(self, table, batch: int):
        if not hasattr(table, "data_ptr"):
            raise TypeError(f"page_table: expected a device tensor, got {type(table).__name__}")
        shape = table.shape
        if table.dtype is not _int32 or len(shape) != 2 or shape[0] != batch or shape[1] < 1:
            raise ValueError(f"page_table: tensor is {tuple(shape)} of {table.dtype}, expected [{batch}, width] of torch.int32")
        if table.get_device() != self._device:
            raise ValueError(f"page_table: tensor is not on device {self._device}")
        width, (apart, element) = shape[1], table.stride()
        if batch < 2:
            apart = width
        if (width > 1 and element != 1) or apart < width:
            raise ValueError("page_table: the entries of a sequence do not lie side by side")
        return table.data_ptr(), width, apart

    def _places(self, cu_seqlens, starts, page_table, tokens: int) -> bytes:
        batch = _count(cu_seqlens, "cu_seqlens") - 1
        if batch < 1:
            raise ValueError("cu_seqlens: expected at least two bounds")
        at, width, stride = self._table(page_table, batch)
        return _PLACES.pack(batch, tokens, ints(cu_seqlens, "cu_seqlens", batch + 1, self._device), ints(starts, "starts", batch, self._device),
                            at, width, stride)

    def append(self, pool, q, k, v, rotation, cu_seqlens, starts, page_table, q_out, k_out, stream: int = 0) -> None:
        """Rotates the packed tokens' q and k into q_out and k_out, and puts keys and values into their pages.
        q, q_out: [tokens, heads, head_dim], both or neither; k, v: [tokens, kv_heads, head_dim]; k_out like k, or None;
        rotation: float32 device tensor [positions, rotary_dim], see rotation_table()."""
        tokens = _count(k, "k")
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out go together")
        if not hasattr(rotation, "data_ptr"):
            raise TypeError(f"rotation: expected a device tensor, got {type(rotation).__name__}")
        if rotation.dtype is not _float32 or rotation.dim() != 2 or rotation.shape[1] != self._rotary or not rotation.is_contiguous():
            raise ValueError(f"rotation: tensor is {tuple(rotation.shape)} of {rotation.dtype}, expected contiguous [positions, {self._rotary}] of torch.float32")
        if rotation.get_device() != self._device:
            raise ValueError(f"rotation: tensor is not on device {self._device}")
        places = self._places(cu_seqlens, starts, page_table, tokens)
        self._check(self.lib.ftcache_append(
            self.handle, self._pool(pool), places, rotation.data_ptr(), rotation.shape[0],
            _NONE if q is None else rows(q, "q", tokens, *self._q), rows(k, "k", tokens, *self._kv), rows(v, "v", tokens, *self._kv),
            _NONE if q_out is None else rows(q_out, "q_out", tokens, *self._q, True),
            _NONE if k_out is None else rows(k_out, "k_out", tokens, *self._kv, True), stream))

    def read(self, pool, k, v, cu_seqlens, starts, page_table, stream: int = 0) -> None:
        """The cached keys and values of the given places into k and v, [tokens, kv_heads, head_dim]."""
        tokens = _count(k, "k")
        places = self._places(cu_seqlens, starts, page_table, tokens)
        self._check(self.lib.ftcache_read(self.handle, self._pool(pool), places, rows(k, "k", tokens, *self._kv, True),
                                          rows(v, "v", tokens, *self._kv, True), stream))

    def attend(self, pool, q, o, lengths, page_table, stream: int = 0) -> None:
        """Attention of one token per sequence, q and o [batch, heads, head_dim], over the first lengths[b] cached tokens."""
        batch = _count(q, "q")
        at, width, stride = self._table(page_table, batch)
        self._check(self.lib.ftcache_attend(self.handle, self._pool(pool), batch, ints(lengths, "lengths", batch, self._device), at, width,
                                            stride, rows(q, "q", batch, *self._q), rows(o, "o", batch, *self._o), stream))

    def report(self):
        """(refused tokens, refused sequences) since the last report; waits for the device."""
        view = ReportView()
        self._check(self.lib.ftcache_report(self.handle, C.byref(view)))
        return int(view.refused_tokens), int(view.refused_sequences)

    def close(self) -> None:
        if self.handle:
            self.lib.ftcache_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
