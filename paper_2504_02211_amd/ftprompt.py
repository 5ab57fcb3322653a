"""Thin ctypes binding of attention over packed prompts in libftattn.so: argument marshalling only.

It raises if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

from . import ftattn as _base

F16, BF16, F32 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4

EXPORTS = ("ftprompt_create", "ftprompt_get_config", "ftprompt_forward", "ftprompt_destroy", "ftprompt_last_error")


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("in_dtype", C.c_int32), ("out_dtype", C.c_int32), ("softmax_scale", C.c_float), ("device", C.c_int32)]


_typed = False
_int32 = None          # torch's, once load_library has run


class FtPromptError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ftprompt error {code}: {msg}")
        self.code = code


def load_library() -> C.CDLL:
    """The shared library with the ftprompt_* prototypes set; raises if it is not built."""
    global _typed, _int32
    lib = _base.load_library()
    if not _typed:
        import torch
        _int32 = torch.int32
        lib.ftprompt_create.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
        lib.ftprompt_get_config.argtypes = [C.c_void_p, C.POINTER(Config)]
        lib.ftprompt_forward.argtypes = [C.c_void_p] * 7 + [C.c_int32] * 3 + [C.c_void_p]
        lib.ftprompt_destroy.argtypes = [C.c_void_p]
        lib.ftprompt_last_error.argtypes = [C.c_void_p]
        lib.ftprompt_last_error.restype = C.c_char_p
        for n in EXPORTS:
            if n != "ftprompt_last_error":
                getattr(lib, n).restype = C.c_int
        _typed = True
    return lib


_ROWS = struct.Struct("=qqq")          # ftprompt_rows and ftcache_rows: address, token stride, head stride


def rows(t, name: str, tokens: int, heads: int, head_dim: int, dtype: int, device: int, out: bool = False) -> bytes:
    """The C structure of a tensor [tokens, heads, head_dim].  Elements of a head lie side by side; the strides of tokens and heads are
    free, those of a result not 0.  A tensor of another size, type or device would be an access out of bounds on the GPU, which the library
    cannot see, so it is refused here.  The ordinary tensor passes all checks in the cheapest way: 0.5 us where the general form takes 0.7."""
    if (heads > 1 and isinstance(t, _base._torch_tensor) and t.dtype is _base._torch_dtype[dtype] and t.get_device() == device
            and t.shape == (tokens, heads, head_dim)):
        token, head, element = t.stride()
        if tokens < 2:
            token = heads * head_dim
        if element == 1 and (not out or (token and head)):
            return _ROWS.pack(t.data_ptr(), token, head)
    if not hasattr(t, "data_ptr"):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != head_dim or shape[0] != tokens:
        raise ValueError(f"{name}: tensor is {tuple(shape)}, expected [{tokens}, {heads}, {head_dim}]")
    if t.dtype is not _base._torch_dtype.get(dtype):
        raise ValueError(f"{name}: tensor is {t.dtype}, expected {_base._TORCH_NAME[dtype]}")
    if not t.is_cuda:
        raise ValueError(f"{name}: tensor is not on a GPU")
    if t.get_device() != device:
        raise ValueError(f"{name}: tensor is on device {t.get_device()}, the context on device {device}")
    if stride[2] != 1:
        raise ValueError(f"{name}: the elements of a head do not lie side by side")
    # (the stride of an axis with one entry says nothing)
    token, head = stride[0] if shape[0] > 1 else heads * head_dim, stride[1] if heads > 1 else head_dim
    if out and (token == 0 or head == 0):
        raise ValueError(f"{name}: a result whose rows lie on one another")
    return _ROWS.pack(t.data_ptr(), token, head)


def ints(t, name: str, n: int, device: int) -> int:
    """Address of a contiguous int32 device tensor of n elements."""
    if isinstance(t, _base._torch_tensor) and t.dtype is _int32 and t.get_device() == device and t.is_contiguous() and t.numel() == n:
        return t.data_ptr()
    if not hasattr(t, "data_ptr"):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}")
    if t.dtype is not _int32:
        raise ValueError(f"{name}: tensor is {t.dtype}, expected torch.int32")
    if not t.is_cuda:
        raise ValueError(f"{name}: tensor is not on a GPU")
    if t.get_device() != device:
        raise ValueError(f"{name}: tensor is on device {t.get_device()}, the context on device {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensor is not contiguous")
    raise ValueError(f"{name}: tensor has {t.numel()} elements, expected {n}")


def array(t, name: str, n: int, dtype, device: int) -> int:
    """Address of a contiguous device tensor of n elements of a torch type."""
    if isinstance(t, _base._torch_tensor) and t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.numel() == n:
        return t.data_ptr()
    if not hasattr(t, "data_ptr"):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: tensor is {t.dtype}, expected {dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name}: tensor is not on a GPU")
    if t.get_device() != device:
        raise ValueError(f"{name}: tensor is on device {t.get_device()}, the context on device {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensor is not contiguous")
    raise ValueError(f"{name}: tensor has {t.numel()} elements, expected {n}")


class FtPrompt:
    """One context of the C library: causal attention of packed sequences for one set of heads on one device."""

    def __init__(self, heads: int, kv_heads: int, head_dim: int, in_dtype: int, out_dtype: Optional[int] = None,
                 softmax_scale: float = 0.0, device: int = 0):
        self.handle = C.c_void_p()
        self.lib = load_library()
        cfg = Config(C.sizeof(Config), heads, kv_heads, head_dim, in_dtype, in_dtype if out_dtype is None else out_dtype,
                     softmax_scale, device)
        rc = self.lib.ftprompt_create(C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            raise FtPromptError(rc, self.lib.ftprompt_last_error(None).decode())
        self.config = Config()
        self.lib.ftprompt_get_config(self.handle, C.byref(self.config))
        e = self.config
        self._q = (e.heads, e.head_dim, e.in_dtype, e.device)
        self._kv = (e.kv_heads, e.head_dim, e.in_dtype, e.device)
        self._o = (e.heads, e.head_dim, e.out_dtype, e.device, True)
        self._device = e.device
        self._forward = self.lib.ftprompt_forward

    def forward(self, q, k, v, o, cu_q, cu_k=None, stream: int = 0) -> None:
        """q, o: [total_q, heads, head_dim], k, v: [total_k, kv_heads, head_dim] device tensors, views of a fused projection among them;
        cu_q, cu_k: int32 device tensors [batch + 1] of row bounds, cu_k None: the same as cu_q."""
        try:
            total_q, total_k, batch = q.shape[0], k.shape[0], cu_q.numel() - 1
        except (AttributeError, IndexError):
            raise TypeError("q, k, cu_q: expected device tensors") from None
        if batch < 1:
            raise ValueError("cu_q: expected at least two bounds")
        at_q = ints(cu_q, "cu_q", batch + 1, self._device)
        at_k = at_q if cu_k is None else ints(cu_k, "cu_k", batch + 1, self._device)
        rc = self._forward(self.handle, rows(q, "q", total_q, *self._q), rows(k, "k", total_k, *self._kv), rows(v, "v", total_k, *self._kv),
                           rows(o, "o", total_q, *self._o), at_q, at_k, batch, total_q, total_k, stream)
        if rc != OK:
            raise FtPromptError(rc, self.lib.ftprompt_last_error(self.handle).decode())

    def close(self) -> None:
        if self.handle:
            self.lib.ftprompt_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
