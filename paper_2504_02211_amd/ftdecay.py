"""Thin ctypes binding of linear attention with a decay for each head in libftattn.so: argument marshalling only.

It raises if the library has not been built -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C

from . import ftattn as _base
from .ftprompt import array, ints, rows

F16, BF16 = 0, 1
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM = 0, -1, -2, -3, -4

EXPORTS = ("ftdecay_create", "ftdecay_get_config", "ftdecay_forward", "ftdecay_step", "ftdecay_destroy", "ftdecay_last_error")


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("in_dtype", C.c_int32),
                ("scale", C.c_float), ("device", C.c_int32)]


_typed = False
_float32 = None          # torch's, once load_library has run


class FtDecayError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ftdecay error {code}: {msg}")
        self.code = code


def load_library() -> C.CDLL:
    """The shared library with the ftdecay_* prototypes set; raises if it is not built."""
    global _typed, _float32
    lib = _base.load_library()
    if not _typed:
        import torch

        from . import ftprompt
        ftprompt.load_library()          # (whose checks of tensors are used here)
        _float32 = torch.float32
        p, i = C.c_void_p, C.c_int32
        lib.ftdecay_create.argtypes = [C.POINTER(Config), C.POINTER(p)]
        lib.ftdecay_get_config.argtypes = [p, C.POINTER(Config)]
        lib.ftdecay_forward.argtypes = [p] * 7 + [i] + [p] * 3 + [i, i, p]
        lib.ftdecay_step.argtypes = [p] * 7 + [i, p, i, p]
        lib.ftdecay_destroy.argtypes = [p]
        lib.ftdecay_last_error.argtypes = [p]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int
        lib.ftdecay_last_error.restype = C.c_char_p
        _typed = True
    return lib


class FtDecay:
    """One context of the C library: linear attention for one set of heads on one device.

    states: a contiguous float32 device tensor [slots, heads, head_dim, head_dim], the caller's; log_decay: float32 [heads]; slots, starts: int32 [batch]."""

    def __init__(self, heads: int, kv_heads: int, head_dim: int, in_dtype: int, scale: float = 0.0, device: int = 0):
        self.handle = C.c_void_p()
        self.lib = load_library()
        cfg = Config(C.sizeof(Config), heads, kv_heads, head_dim, in_dtype, scale, device)
        rc = self.lib.ftdecay_create(C.byref(cfg), C.byref(self.handle))
        if rc != OK:
            self.handle = C.c_void_p()
            raise FtDecayError(rc, self.lib.ftdecay_last_error(None).decode())
        self.config = Config()
        self.lib.ftdecay_get_config(self.handle, C.byref(self.config))
        e = self.config
        self._q = (e.heads, e.head_dim, e.in_dtype, e.device)
        self._kv = (e.kv_heads, e.head_dim, e.in_dtype, e.device)
        self._o = (*self._q, True)
        self._heads, self._state, self._device = e.heads, e.heads * e.head_dim * e.head_dim, e.device

    def _check(self, rc: int) -> None:
        if rc != OK:
            raise FtDecayError(rc, self.lib.ftdecay_last_error(self.handle).decode())

    def _states(self, states, slots, batch: int):
        """(address of the pool, its slots, address of the sequences' slots)"""
        if not hasattr(states, "data_ptr"):
            raise TypeError(f"states: expected a device tensor, got {type(states).__name__}")
        n = states.numel() // self._state
        at = array(states, "states", n * self._state, _float32, self._device)
        if slots is None and n < batch:
            raise ValueError(f"states: room for {n} sequences, expected {batch}")
        return at, n, None if slots is None else ints(slots, "slots", batch, self._device)

    def forward(self, q, k, v, o, log_decay, states, cu, starts=None, slots=None, stream: int = 0) -> None:
        """q, o: [total, heads, head_dim], k, v: [total, kv_heads, head_dim] device tensors, views of a fused projection among them; cu: int32
        [batch + 1] of row bounds; starts: tokens that a sequence had before these (0: it begins with zeros), None: all begin; slots: where the
        sequences' states lie, None: in their order; states None: none are kept."""
        try:
            total, batch = q.shape[0], cu.numel() - 1
        except (AttributeError, IndexError):
            raise TypeError("q, cu: expected device tensors") from None
        if batch < 1:
            raise ValueError("cu: expected at least two bounds")
        at, n, where = (None, 0, None) if states is None else self._states(states, slots, batch)
        self._check(self.lib.ftdecay_forward(
            self.handle, rows(q, "q", total, *self._q), rows(k, "k", total, *self._kv), rows(v, "v", total, *self._kv), rows(o, "o", total, *self._o),
            array(log_decay, "log_decay", self._heads, _float32, self._device), at, n, where, ints(cu, "cu", batch + 1, self._device),
            None if starts is None else ints(starts, "starts", batch, self._device), batch, total, stream))

    def step(self, q, k, v, o, log_decay, states, slots=None, stream: int = 0) -> None:
        """One token of every sequence: q, o [batch, heads, head_dim], k, v [batch, kv_heads, head_dim]; every state moves on by it."""
        try:
            batch = q.shape[0]
        except (AttributeError, IndexError):
            raise TypeError("q: expected a device tensor") from None
        at, n, where = self._states(states, slots, batch)
        self._check(self.lib.ftdecay_step(
            self.handle, rows(q, "q", batch, *self._q), rows(k, "k", batch, *self._kv), rows(v, "v", batch, *self._kv), rows(o, "o", batch, *self._o),
            array(log_decay, "log_decay", self._heads, _float32, self._device), at, n, where, batch, stream))

    def close(self) -> None:
        if self.handle:
            self.lib.ftdecay_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
