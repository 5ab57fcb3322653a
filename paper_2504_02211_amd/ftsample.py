"""Thin ctypes binding of the choice of the next token in libftattn.so: argument marshalling only.

It raises if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import struct

from . import ftattn as _base
from .ftprompt import array

F16, BF16, F32 = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4

EXPORTS = ("ftsample_create", "ftsample_get_config", "ftsample_choose", "ftsample_destroy", "ftsample_last_error")


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("vocab", C.c_int32), ("max_rows", C.c_int32), ("in_dtype", C.c_int32), ("device", C.c_int32)]


_typed = False
_int32 = _float32 = None          # torch's, once load_library has run


class FtSampleError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ftsample error {code}: {msg}")
        self.code = code


def load_library() -> C.CDLL:
    """The shared library with the ftsample_* prototypes set; raises if it is not built."""
    global _typed, _int32, _float32
    lib = _base.load_library()
    if not _typed:
        import torch
        _int32, _float32 = torch.int32, torch.float32
        p = C.c_void_p
        lib.ftsample_create.argtypes = [C.POINTER(Config), C.POINTER(p)]
        lib.ftsample_get_config.argtypes = [p, C.POINTER(Config)]
        lib.ftsample_choose.argtypes = [p, p, C.c_int64, C.c_int32, p, p, p, p, p]
        lib.ftsample_destroy.argtypes = [p]
        lib.ftsample_last_error.argtypes = [p]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        lib.ftsample_last_error.restype = C.c_char_p
        _typed = True
    return lib


_RULES = struct.Struct("@PPPP")          # ftsample_rules


class FtSample:
    """One context of the C library: rows of logits of one vocabulary and type on one device."""

    def __init__(self, vocab: int, in_dtype: int, max_rows: int = 256, device: int = 0):
        self.handle = C.c_void_p()
        self.lib = load_library()
        cfg = Config(C.sizeof(Config), vocab, max_rows, in_dtype, device)
        rc = self.lib.ftsample_create(C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            raise FtSampleError(rc, self.lib.ftsample_last_error(None).decode())
        self.config = Config()
        self.lib.ftsample_get_config(self.handle, C.byref(self.config))
        e = self.config
        self._vocab, self._dtype, self._device = e.vocab, _base._torch_dtype[e.in_dtype], e.device

    def choose(self, logits, uniform, tokens, temperature=None, top_k=None, top_p=None, min_p=None, probability=None, stream: int = 0) -> None:
        """The next token of every row of logits [rows, vocab] (rows may lie apart) from one random number of [0, 1) per row into tokens, int32 [rows];
        probability, float32 [rows] or None: its share of the kept weights.  temperature, top_p, min_p (float32 [rows]) and top_k (int32 [rows]):
        the rules of each row, or None."""
        if not isinstance(logits, _base._torch_tensor):
            raise TypeError(f"logits: expected a device tensor, got {type(logits).__name__}")
        shape, device = logits.shape, self._device
        if len(shape) != 2 or shape[1] != self._vocab:
            raise ValueError(f"logits: tensor is {tuple(shape)}, expected [rows, {self._vocab}]")
        if logits.dtype is not self._dtype:
            raise ValueError(f"logits: tensor is {logits.dtype}, expected {self._dtype}")
        if logits.get_device() != device:
            raise ValueError(f"logits: tensor is not on device {device}")
        n, (apart, element) = shape[0], logits.stride()
        if element != 1 and self._vocab > 1:
            raise ValueError("logits: the elements of a row do not lie side by side")
        numbers = lambda t, name: 0 if t is None else array(t, name, n, _float32, device)  # noqa: E731
        rules = _RULES.pack(numbers(temperature, "temperature"), 0 if top_k is None else array(top_k, "top_k", n, _int32, device),
                            numbers(top_p, "top_p"), numbers(min_p, "min_p"))
        rc = self.lib.ftsample_choose(self.handle, logits.data_ptr(), apart if n > 1 else 0, n, array(uniform, "uniform", n, _float32, device), rules,
                                      array(tokens, "tokens", n, _int32, device), numbers(probability, "probability") or None, stream)
        if rc != OK:
            raise FtSampleError(rc, self.lib.ftsample_last_error(self.handle).decode())

    def close(self) -> None:
        if self.handle:
            self.lib.ftsample_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
