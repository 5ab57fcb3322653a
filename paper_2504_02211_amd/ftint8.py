"""Thin ctypes binding of the linear layer on 8-bit integers in libftattn.so: argument marshalling only.

It raises if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

from . import ftattn as _base
from .ftprompt import array

F16, BF16, F32 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4

EXPORTS = ("ftint8_create", "ftint8_get_config", "ftint8_k_padded", "ftint8_encode", "ftint8_product", "ftint8_forward", "ftint8_destroy",
           "ftint8_last_error")


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n", C.c_int32), ("k", C.c_int32), ("in_dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("max_tokens", C.c_int32), ("device", C.c_int32)]


_typed = False
_int8 = _float32 = None          # torch's, once load_library has run


class FtInt8Error(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ftint8 error {code}: {msg}")
        self.code = code


def load_library() -> C.CDLL:
    """The shared library with the ftint8_* prototypes set; raises if it is not built."""
    global _typed, _int8, _float32
    lib = _base.load_library()
    if not _typed:
        import torch
        _int8, _float32 = torch.int8, torch.float32
        p, i = C.c_void_p, C.c_int32
        lib.ftint8_create.argtypes = [C.POINTER(Config), C.POINTER(p)]
        lib.ftint8_get_config.argtypes = [p, C.POINTER(Config)]
        lib.ftint8_k_padded.argtypes = [p]
        lib.ftint8_encode.argtypes = [p, p, i, p, p, p]
        lib.ftint8_product.argtypes = [p, p, p, i, p, p, p, p]
        lib.ftint8_forward.argtypes = [p, p, i, p, p, p, p]
        lib.ftint8_destroy.argtypes = [p]
        lib.ftint8_last_error.argtypes = [p]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        lib.ftint8_last_error.restype = C.c_char_p
        _typed = True
    return lib


_MATRIX = struct.Struct("=qq")          # ftint8_matrix: address, stride


def matrix(t, name: str, columns: int, dtype: int, device: int) -> bytes:
    """The C structure of a tensor [rows, columns] whose rows may lie apart.  A tensor of another size, type or device would be an access out of
    bounds on the GPU, which the library cannot see, so it is refused here."""
    if not isinstance(t, _base._torch_tensor):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}")
    shape = t.shape
    if len(shape) != 2 or shape[1] != columns:
        raise ValueError(f"{name}: tensor is {tuple(shape)}, expected [rows, {columns}]")
    if t.dtype is not _base._torch_dtype[dtype]:
        raise ValueError(f"{name}: tensor is {t.dtype}, expected {_base._TORCH_NAME[dtype]}")
    at = t.get_device()
    if at < 0:
        raise ValueError(f"{name}: tensor is not on a GPU")
    if at != device:
        raise ValueError(f"{name}: tensor is on device {at}, the context on device {device}")
    apart, element = t.stride()
    if element != 1 and columns > 1:
        raise ValueError(f"{name}: the elements of a row do not lie side by side")
    # (the stride of an axis with one entry says nothing)
    if shape[0] < 2:
        apart = columns
    elif apart < columns:
        raise ValueError(f"{name}: rows that lie on one another")
    return _MATRIX.pack(t.data_ptr(), apart)


def _rows(t, name: str) -> int:
    try:
        return t.shape[0]
    except (AttributeError, IndexError):
        raise TypeError(f"{name}: expected a device tensor, got {type(t).__name__}") from None


class FtInt8:
    """One context of the C library: layers of n output and k input features on one device.

    Codes are contiguous int8 device tensors [rows, k_padded] (k rounded up to a multiple of 128, zeros behind column k), scales float32 [rows]."""

    def __init__(self, n: int, k: int, in_dtype: int, out_dtype: Optional[int] = None, max_tokens: int = 1, device: int = 0):
        self.handle = C.c_void_p()
        self.lib = load_library()
        cfg = Config(C.sizeof(Config), n, k, in_dtype, in_dtype if out_dtype is None else out_dtype, max_tokens, device)
        rc = self.lib.ftint8_create(C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            raise FtInt8Error(rc, self.lib.ftint8_last_error(None).decode())
        self.config = Config()
        self.lib.ftint8_get_config(self.handle, C.byref(self.config))
        e = self.config
        self.k_padded = self.lib.ftint8_k_padded(self.handle)
        self._x, self._y, self._device = (e.k, e.in_dtype, e.device), (e.n, e.out_dtype, e.device), e.device
        self._n, self._codes = e.n, e.n * self.k_padded

    def _check(self, rc: int) -> None:
        if rc != OK:
            raise FtInt8Error(rc, self.lib.ftint8_last_error(self.handle).decode())

    def encode(self, x, codes, scales, stream: int = 0) -> None:
        """Codes and scales of the rows of x [rows, k]: of weights, or of tokens that several layers read."""
        rows = _rows(x, "x")
        self._check(self.lib.ftint8_encode(self.handle, matrix(x, "x", *self._x), rows, array(codes, "codes", rows * self.k_padded, _int8, self._device),
                                           array(scales, "scales", rows, _float32, self._device), stream))

    def product(self, codes_x, scales_x, codes_w, scales_w, y, stream: int = 0) -> None:
        """y [m, n] from the codes and scales of m tokens and of the layer's n channels."""
        m = _rows(y, "y")
        self._check(self.lib.ftint8_product(
            self.handle, array(codes_x, "codes_x", m * self.k_padded, _int8, self._device), array(scales_x, "scales_x", m, _float32, self._device), m,
            array(codes_w, "codes_w", self._codes, _int8, self._device), array(scales_w, "scales_w", self._n, _float32, self._device),
            matrix(y, "y", *self._y), stream))

    def forward(self, x, codes_w, scales_w, y, stream: int = 0) -> None:
        """y [m, n] from m <= max_tokens tokens x [m, k] in 16 bits."""
        m = _rows(x, "x")
        if _rows(y, "y") != m:
            raise ValueError(f"y: tensor is {tuple(y.shape)}, x {tuple(x.shape)}")
        self._check(self.lib.ftint8_forward(self.handle, matrix(x, "x", *self._x), m, array(codes_w, "codes_w", self._codes, _int8, self._device),
                                            array(scales_w, "scales_w", self._n, _float32, self._device), matrix(y, "y", *self._y), stream))

    def close(self) -> None:
        if self.handle:
            self.lib.ftint8_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
