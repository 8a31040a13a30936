"""The 4-bit key / value cache of libs2d2.so (include/s2d2_kv4.h) on torch tensors: argument marshalling only.

A `Kv4Cache` owns the tensors of a cache and can stand in for a `KvCache` in the calls of an `Engine` whose context it is
attached to (`s2d2_set_kv4`); the functions below are the C calls that need no context.  They run on the given stream, by
default the current one of the cache's device.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import S2D2_BF16, S2D2_EINVAL, S2D2_F32, KvView, S2D2Error, _check, _ptr, load_library

EXPORTS = ["s2d2_kv4_append", "s2d2_kv4_read", "s2d2_kv4_attention_bytes", "s2d2_kv4_attention", "s2d2_kv4_weigh", "s2d2_kv4_evict_bytes", "s2d2_kv4_evict", "s2d2_set_kv4"]
GROUP = 32   # values that share a power of two


class Kv4View(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scales", "v_scales", "mass", "position", "page_table", "entries",
                                          "seq_len", "status")] + \
               [(n, C.c_int32) for n in ("n_layers", "n_pages", "page_size", "max_pages_per_seq", "n_kv_heads", "head_dim")]


class Kv4RowsC(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("N", "T", "rows", "n_q_heads", "dtype")] + [("scale", C.c_float)] + \
               [(n, C.c_void_p) for n in ("q", "k", "v")] + [(n, C.c_int64) for n in ("q_stride", "kv_stride", "out_stride")] + \
               [(n, C.c_void_p) for n in ("row0", "n_rows", "lo", "hi", "out", "lse")]


_DTYPES = {torch.bfloat16: S2D2_BF16, torch.float32: S2D2_F32}
_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        lib = load_library()
        i32, i64, p = C.c_int32, C.c_int64, C.c_void_p
        view, rows = C.POINTER(Kv4View), C.POINTER(Kv4RowsC)
        lib.s2d2_kv4_append.argtypes = [p, view, i32, i32, i32, i32, p, p, i64, i64, p, p]
        lib.s2d2_kv4_read.argtypes = [p, view, i32, i32, i32, p, p, p]
        lib.s2d2_kv4_attention_bytes.argtypes = [view, i32, i32, i32]
        lib.s2d2_kv4_attention.argtypes = [p, view, i32, rows, p, C.c_size_t]
        lib.s2d2_kv4_weigh.argtypes = [p, view, i32, rows]
        lib.s2d2_kv4_evict_bytes.argtypes = [view, i32]
        lib.s2d2_kv4_evict.argtypes = [p, view, i32, i32, i32, i32, i32, p, C.c_size_t]
        lib.s2d2_set_kv4.argtypes = [p, view, p, C.c_size_t, p]
        for n in EXPORTS:
            getattr(lib, n).restype = C.c_int64 if n.endswith("_bytes") else C.c_int32
        _LIB = lib
    return _LIB


def _refuse(why: str):
    raise S2D2Error(S2D2_EINVAL, why)


def _need(t: Optional[torch.Tensor], name: str, shape, dtype, device):
    """A contiguous tensor of this shape and type on this device."""
    if t is None:
        _refuse(f"{name} is missing")
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rows_layout(t: torch.Tensor, name: str, rows: int, heads: int, dim: int, dtype, device) -> int:
    """[rows, heads, dim] with whole rows, any distance apart: the row stride in elements."""
    if t.shape != (rows, heads, dim) or t.dtype != dtype or t.device != device:
        _refuse(f"{name} must be a {dtype} tensor of shape {(rows, heads, dim)} on {device}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != dim):
        _refuse(f"{name}: the heads of a row must lie one behind the other, strides are {t.stride()}")
    return t.stride(0) if rows > 1 else heads * dim


class Kv4Cache:
    """k_codes, v_codes uint8 [n_layers, n_pages, Hkv, page_size, D / 2]; k_scales, v_scales uint8 [.., D / 32]; mass fp32 and position int32
    [n_layers, n_pages, Hkv, page_size] or None (both: an eviction scratch of 4 bytes a place and list comes with them); page_table int32 [N, max_pages]; entries, seq_len, status int32 [N]."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales, page_table, entries, seq_len, status=None, mass=None, position=None):
        if k_codes.dim() != 5 or k_codes.dtype != torch.uint8:
            _refuse("k_codes must be uint8 [n_layers, n_pages, n_kv_heads, page_size, head_dim / 2]")
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, half = k_codes.shape
        self.head_dim, self.device = 2 * half, k_codes.device
        if self.device.type != "cuda":
            _refuse("a 4-bit cache lives on a GPU")
        shape = tuple(k_codes.shape[:4])
        for t, name, last, dtype in ((k_codes, "k_codes", (half,), torch.uint8), (v_codes, "v_codes", (half,), torch.uint8),
                                     (k_scales, "k_scales", (self.head_dim // GROUP,), torch.uint8), (v_scales, "v_scales", (self.head_dim // GROUP,), torch.uint8),
                                     (mass, "mass", (), torch.float32), (position, "position", (), torch.int32)):
            if t is not None or name not in ("mass", "position"):
                _need(t, name, shape + last, dtype, self.device)
        if page_table.dim() != 2:
            _refuse("page_table must be int32 [N, max_pages_per_seq]")
        self.N = page_table.shape[0]
        _need(page_table, "page_table", page_table.shape, torch.int32, self.device)
        for t, name in ((entries, "entries"), (seq_len, "seq_len"), (status, "status")):
            if t is not None or name != "status":
                _need(t, name, (self.N,), torch.int32, self.device)
        self.k_codes, self.v_codes, self.k_scales, self.v_scales = k_codes, v_codes, k_scales, v_scales
        self.mass, self.position, self.page_table, self.entries, self.seq_len, self.status = mass, position, page_table, entries, seq_len, status
        self._view = Kv4View(*[_ptr(t) for t in (k_codes, v_codes, k_scales, v_scales, mass, position, page_table, entries, seq_len, status)],
                             self.n_layers, self.n_pages, self.page_size, page_table.shape[1], self.n_kv_heads, self.head_dim)
        self._ref = C.byref(self._view)
        self.moves = None   # scratch of the eviction, with mass and position
        if mass is not None and position is not None:
            n = _lib().s2d2_kv4_evict_bytes(self._ref, self.N)
            if n < 0:
                raise S2D2Error(int(n), _LIB.s2d2_last_error().decode())
            self.moves = torch.empty(int(n), dtype=torch.uint8, device=self.device)

    @staticmethod
    def alloc(n_layers: int, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, page_table: torch.Tensor, weights: bool = False) -> "Kv4Cache":
        """An empty cache behind this page table; weights: with mass and position, as eviction needs them."""
        dev, shape = page_table.device, (n_layers, n_pages, n_kv_heads, page_size)
        byte = lambda last: torch.zeros((*shape, last), dtype=torch.uint8, device=dev)  # noqa: E731
        word = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
        n = page_table.shape[0]
        return Kv4Cache(byte(head_dim // 2), byte(head_dim // 2), byte(head_dim // GROUP), byte(head_dim // GROUP), page_table, word(n), word(n), word(n),
                        torch.zeros(shape, device=dev) if weights else None, word(shape) if weights else None)

    def c(self) -> KvView:
        """The view that the calls of an Engine take while this cache is attached to its context."""
        return KvView(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.page_table.data_ptr(), self.seq_len.data_ptr(), _ptr(self.status),
                      self.n_pages, self.page_size, self.page_table.shape[1])

    def _stream(self, stream: Optional[torch.cuda.Stream]) -> int:
        return (stream if stream is not None else torch.cuda.current_stream(self.device)).cuda_stream

    def _call(self, fn, stream, *args):
        if torch.cuda.current_device() == self.device.index:
            _check(_LIB, fn(self._stream(stream), self._ref, *args))
        else:
            with torch.cuda.device(self.device):
                _check(_LIB, fn(self._stream(stream), self._ref, *args))


class Kv4Rows:
    """Windows of N sequences (s2d2_kv4_rows): q, out [rows, Hq, D]; k, v [rows, Hkv, D] or None; row0, n_rows int32 [N]; lo, hi int32 [rows] or None;
    lse fp32 [rows, Hq] or None; T: most rows of a sequence."""

    def __init__(self, q, row0, n_rows, T: int, scale: float, out=None, lse=None, k=None, v=None, lo=None, hi=None):
        if q.dim() != 3 or q.dtype not in _DTYPES:
            _refuse("q must be a bf16 or fp32 tensor [rows, n_q_heads, head_dim]")
        rows, hq, dim = q.shape
        dev = q.device
        q_ld = _rows_layout(q, "q", rows, hq, dim, q.dtype, dev)
        o_ld = _rows_layout(out, "out", rows, hq, dim, q.dtype, dev) if out is not None else 0
        if (k is None) != (v is None) or (lo is None) != (hi is None):
            _refuse("k and v, and lo and hi, are given together or not at all")
        kv_ld = 0
        if k is not None:
            kv_ld, v_ld = _rows_layout(k, "k", rows, k.shape[1], dim, q.dtype, dev), _rows_layout(v, "v", rows, k.shape[1], dim, q.dtype, dev)
            if kv_ld != v_ld:
                _refuse("k and v must have the same row stride")
        N = row0.shape[0]
        _need(row0, "row0", (N,), torch.int32, dev)
        _need(n_rows, "n_rows", (N,), torch.int32, dev)
        for t, name, shape, dtype in ((lo, "lo", (rows,), torch.int32), (hi, "hi", (rows,), torch.int32), (lse, "lse", (rows, hq), torch.float32)):
            if t is not None:
                _need(t, name, shape, dtype, dev)
        self.kv_heads = None if k is None else k.shape[1]
        self.head_dim, self.device, self.n = dim, dev, N
        self.tensors = (q, k, v, row0, n_rows, lo, hi, out, lse)   # (alive as long as the pointers)
        self.q, self.out, self.lse = q, out, lse
        self._c = Kv4RowsC(N, T, rows, hq, _DTYPES[q.dtype], scale, q.data_ptr(), _ptr(k), _ptr(v), q_ld, kv_ld, o_ld, row0.data_ptr(), n_rows.data_ptr(),
                           _ptr(lo), _ptr(hi), _ptr(out), _ptr(lse))
        self._ref = C.byref(self._c)

    def _fits(self, kv: Kv4Cache):
        if self.device != kv.device or self.head_dim != kv.head_dim or self.n != kv.N or self.kv_heads not in (None, kv.n_kv_heads):
            _refuse(f"rows of {self.n} sequences, {self.kv_heads} KV heads, head_dim {self.head_dim} on {self.device} do not fit a cache of "
                    f"{kv.N}, {kv.n_kv_heads}, {kv.head_dim} on {kv.device}")


def s2d2_kv4_append(kv: Kv4Cache, k: torch.Tensor, v: torch.Tensor, row0: torch.Tensor, n_rows: torch.Tensor, T: int, stream: Optional[torch.cuda.Stream] = None):
    """k, v [n_layers, rows, Hkv, D] in bf16 or fp32, rows any distance apart; row0, n_rows int32 [N]."""
    lib = _LIB or _lib()
    if k.dim() != 4 or k.dtype not in _DTYPES or k.shape[0] != kv.n_layers or v.shape != k.shape or v.stride() != k.stride():
        _refuse(f"k and v must be bf16 or fp32 [n_layers, rows, n_kv_heads, head_dim] of the same strides, not {tuple(k.shape)} and {tuple(v.shape)}")
    ld = 0
    for t, name in ((k, "k"), (v, "v")):
        ld = _rows_layout(t[0], name, k.shape[1], kv.n_kv_heads, kv.head_dim, k.dtype, kv.device)
    _need(row0, "row0", (kv.N,), torch.int32, kv.device)
    _need(n_rows, "n_rows", (kv.N,), torch.int32, kv.device)
    kv._call(lib.s2d2_kv4_append, stream, kv.N, T, k.shape[1], _DTYPES[k.dtype], k.data_ptr(), v.data_ptr(), k.stride(0) if kv.n_layers > 1 else 0, ld,
             row0.data_ptr(), n_rows.data_ptr())


def s2d2_kv4_read(kv: Kv4Cache, first: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
    """Entries first[n] .. into k, v [n_layers, N, T, Hkv, D], bf16 or fp32."""
    lib = _LIB or _lib()
    if k.dim() != 5 or k.dtype not in _DTYPES:
        _refuse("k and v must be bf16 or fp32 [n_layers, N, T, n_kv_heads, head_dim]")
    shape = (kv.n_layers, kv.N, k.shape[2], kv.n_kv_heads, kv.head_dim)
    _need(k, "k", shape, k.dtype, kv.device)
    _need(v, "v", shape, k.dtype, kv.device)
    _need(first, "first", (kv.N,), torch.int32, kv.device)
    kv._call(lib.s2d2_kv4_read, stream, kv.N, k.shape[2], _DTYPES[k.dtype], first.data_ptr(), k.data_ptr(), v.data_ptr())


def s2d2_kv4_attention_bytes(kv: Kv4Cache, N: int, T: int, n_q_heads: int) -> int:
    lib = _LIB or _lib()
    n = lib.s2d2_kv4_attention_bytes(kv._ref, N, T, n_q_heads)
    if n < 0:
        raise S2D2Error(int(n), lib.s2d2_last_error().decode())
    return int(n)


def s2d2_kv4_attention(kv: Kv4Cache, layer: int, rows: Kv4Rows, scratch: torch.Tensor, stream: Optional[torch.cuda.Stream] = None):
    """Writes rows.out (and rows.lse); scratch: uint8, s2d2_kv4_attention_bytes() or more."""
    lib = _LIB or _lib()
    rows._fits(kv)
    if scratch.device != kv.device or not scratch.is_contiguous():
        _refuse(f"scratch must be contiguous on {kv.device}")
    kv._call(lib.s2d2_kv4_attention, stream, layer, rows._ref, scratch.data_ptr(), scratch.numel() * scratch.element_size())


def s2d2_kv4_weigh(kv: Kv4Cache, layer: int, rows: Kv4Rows, stream: Optional[torch.cuda.Stream] = None):
    """Adds the weights of the rows, by their lse, to kv.mass."""
    lib = _LIB or _lib()
    rows._fits(kv)
    kv._call(lib.s2d2_kv4_weigh, stream, layer, rows._ref)


def s2d2_kv4_evict(kv: Kv4Cache, budget: int, slack: int = 0, sink: int = 0, recent: int = 0, stream: Optional[torch.cuda.Stream] = None):
    """Cuts the sequences with more than budget + slack entries to `budget` of them, list by list; the scratch is the cache's own.  Entries of
    s2d2_kv4_append that no rows have been weighed against yet stand at 0: protect them by `recent`."""
    lib = _LIB or _lib()
    moves = kv.moves
    kv._call(lib.s2d2_kv4_evict, stream, kv.N, budget, slack, sink, recent, _ptr(moves), 0 if moves is None else moves.numel())


def _release(held, stream):
    """Scratch and lse of an attachment that ended: their memory is free when the engine's stream is done with them."""
    for t in (held or (None,))[1:]:
        if t is not None:
            t.record_stream(stream)


def s2d2_set_kv4(eng, kv: Optional[Kv4Cache]):
    """Attaches the cache to the engine's context (None: detaches): from now on its calls take `kv` where they take a KvCache."""
    lib = _lib()
    held = getattr(eng, "_kv4", None)
    if kv is None:
        _check(lib, lib.s2d2_set_kv4(eng.ctx, None, None, 0, None))
        eng._kv4 = None
        _release(held, eng.stream)
        return
    if kv.device != torch.device(eng.device.type, eng.device.index or 0) or kv.N > eng.max_batch:
        _refuse(f"a cache of {kv.N} sequences on {kv.device} does not fit an engine of {eng.max_batch} on {eng.device}")
    heads = eng.cfg.n_q_heads
    need = s2d2_kv4_attention_bytes(kv, eng.max_batch, 3 * eng.max_block, heads)
    scratch = torch.empty(need, dtype=torch.uint8, device=kv.device)
    lse = torch.empty(eng.stage_rows, heads, device=kv.device) if kv.mass is not None else None
    _check(lib, lib.s2d2_set_kv4(eng.ctx, kv._ref, scratch.data_ptr(), need, _ptr(lse)))
    eng._kv4 = (kv, scratch, lse)   # alive while the context uses them
    _release(held, eng.stream)
