"""Paged 8-bit KV cache for MI355X: page tables and slot maps built on the GPU,
the append that quantizes keys and values into pages, and attention over them.

Thin ctypes binding of ``libturboesm_paged.so`` (C ABI in
``include/turboesm_paged.h``). Beside the 3-bit cache of the package's root
module it holds e4m3 codes with one power-of-two scale per page of 64 tokens
and head, in pages that any sequence may own; query heads may share key/value
heads, and a sequence may have any number of query tokens. Types are fp16,
bf16 and fp32. If the library is not built, calls raise ``RuntimeError``.

A serving loop:

    pool, cache = paged.PagePool(pages), paged.Cache(L, kv_heads, pages)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    slots, pos, row0, granted = paged.assign(pool, table, seq_len, new_tokens, rows)
    for l in range(L):                     # q, k, v: [1][rows][heads][64], rows of all sequences packed
        paged.append(params, cache, k, v, slots, pos, layer0=l)
        out = paged.attend(params, cache, q, pos, row0, table, seq_len, max_new, max_len, layer0=l)
    paged.release(pool, table, seq_len, keep)     # keep[b] = 0 where a sequence is finished

Every call goes to the current stream of its tensors' device, never
synchronizes, and can be captured into a graph.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

from . import OUT_FP32, ROPE_HALF, TQError, _raw_stream

__all__ = ["Params", "Cache", "PagePool", "assign", "release", "append", "attend", "workspace_bytes", "cache_bytes",
           "last_error", "lib_path", "PAGE", "MAX_SEQS", "ROPE_HALF", "OUT_FP32"]

PAGE, MAX_SEQS = 64, 4096
_IO = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}

lib_path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libturboesm_paged.so")


class _Params(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("num_layers", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("softmax_scale", ctypes.c_float), ("rope_positions", ctypes.c_int32), ("rope_cs", ctypes.c_void_p)]


class _Cache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("pages", ctypes.c_int64)]


class _Pool(ctypes.Structure):
    _fields_ = [("stack", ctypes.c_void_p), ("state", ctypes.c_void_p), ("pages", ctypes.c_int64)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("layer_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


_lib = None


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(lib_path):
        raise RuntimeError(f"{lib_path} is not built; run __graft_entry__.build() "
                           "or python -m paper_2603_26110_amd.build")
    L = ctypes.CDLL(lib_path)
    P, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    L.tqp_last_error.restype = ctypes.c_char_p
    L.tqp_cache_bytes.argtypes = [i32, i32, i64]
    L.tqp_cache_bytes.restype = i64
    L.tqp_assign.argtypes = [P, P, i32, i32, P, P, i32, P, P, P, P, P]
    L.tqp_assign.restype = i32
    L.tqp_release.argtypes = [P, P, i32, i32, P, P, P]
    L.tqp_release.restype = i32
    L.tqp_append.argtypes = [P, P, P, P, i32, i32, i32, P, P, P]
    L.tqp_append.restype = i32
    L.tqp_attend.argtypes = [P, P, P, i32, i32, i32, i32, P, P, P, i32, P, i32, i32, i32, P, P, sz, P]
    L.tqp_attend.restype = i32
    L.tqp_workspace_bytes.argtypes = [P, i32, i32, i32, i32]
    L.tqp_workspace_bytes.restype = sz
    _lib = L
    return L


def last_error() -> str:
    return _load().tqp_last_error().decode()


def _check(status: int) -> None:
    if status != 0:
        raise TQError(f"status {status}: {last_error()}")


def _dev(t, name: str, dtype, device=None, numel: int | None = None) -> torch.Tensor:
    """A contiguous tensor of the type, on `device`, with at least `numel` elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} needs {numel} entries")
    return t


def _rows(t, name: str, dtype, nheads: int, device=None) -> _Rows:
    """A [nlayers][rows][heads][64] tensor of any strides that the library takes."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 4 or t.shape[3] != 64 or t.shape[2] != nheads:
        raise ValueError(f"{name} must be [nlayers][rows][{nheads}][64]")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    s = t.stride()
    if s[3] != 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    # (the stride of a dimension of one entry says nothing)
    return _Rows(t.data_ptr(), *[0 if n == 1 else x for n, x in zip(t.shape[:3], s)])


class _on:
    """The device of a call's tensors as the current one (the library launches there)."""

    def __init__(self, device):
        self.index = device.index

    def __enter__(self):
        self.back = torch.cuda.current_device()
        if self.back != self.index:
            torch.cuda.set_device(self.index)
        return _raw_stream(self.index)

    def __exit__(self, *_):
        if self.back != self.index:
            torch.cuda.set_device(self.back)


@dataclass
class Params:
    """Model-level parameters (tqp_params). ``rope_cs`` comes from the package's
    rope_table(); None where q and k come rotated, or the model has no RoPE."""
    num_layers: int
    num_heads: int
    kv_heads: int
    rope_cs: torch.Tensor | None = None
    io_dtype: torch.dtype = torch.float16
    flags: int = 0
    softmax_scale: float = 0.125

    def c(self, device=None) -> _Params:
        if self.io_dtype not in _IO:
            raise TypeError(f"io_dtype must be one of {[str(d) for d in _IO]}")
        cs = self.rope_cs
        if cs is not None:
            _dev(cs, "rope_cs", torch.float32, device)
            if cs.dim() != 3 or tuple(cs.shape[1:]) != (32, 2):
                raise ValueError("rope_cs must be [positions][32][2]")
        return _Params(64, self.num_layers, self.num_heads, self.kv_heads, _IO[self.io_dtype], self.flags,
                       self.softmax_scale, 0 if cs is None else cs.shape[0], None if cs is None else cs.data_ptr())


class Cache:
    """Pages in device memory: per (layer, key/value head, page) 4096 key codes, 4096 value codes and two scales.
    ``buffers``: the caller's own (k_codes, v_codes, scales) in place of new, zeroed ones."""

    def __init__(self, num_layers: int, kv_heads: int, pages: int, device="cuda", buffers=None):
        if num_layers <= 0 or kv_heads <= 0 or pages <= 0:
            raise ValueError("num_layers, kv_heads and pages must be positive")
        self.num_layers, self.kv_heads, self.pages = num_layers, kv_heads, pages
        shape = (num_layers, kv_heads, pages)
        if buffers is None:
            self.k_codes = torch.zeros((*shape, PAGE * 64), dtype=torch.uint8, device=device)
            self.v_codes = torch.zeros((*shape, PAGE * 64), dtype=torch.uint8, device=device)
            self.scales = torch.full((*shape, 2), 2.0 ** -48, dtype=torch.float32, device=device)
        else:
            self.k_codes, self.v_codes, self.scales = buffers
            for name, t, last in (("k_codes", self.k_codes, PAGE * 64), ("v_codes", self.v_codes, PAGE * 64),
                                  ("scales", self.scales, 2)):
                _dev(t, name, torch.float32 if last == 2 else torch.uint8, self.k_codes.device)
                if tuple(t.shape) != (*shape, last):
                    raise ValueError(f"{name} must be {[*shape, last]}")
        self.device = self.k_codes.device
        self._c = _Cache(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.scales.data_ptr(), pages)

    def values(self):
        """Views of what the cache holds, as float8_e4m3fn tensors: keys [L][kv_heads][pages][64 tokens][64], values
        [L][kv_heads][pages][4][4][4][64] (token 16 i + 4 g + r at [i][g][r]), and the scales [L][kv_heads][pages][2]
        of keys and values that they are multiplied by."""
        shape = (self.num_layers, self.kv_heads, self.pages)
        k = self.k_codes.view(torch.float8_e4m3fn).view(*shape, PAGE, 64)
        v = self.v_codes.view(torch.float8_e4m3fn).view(*shape, 4, 64, 4, 4).permute(0, 1, 2, 5, 3, 6, 4)
        return k, v, self.scales


class PagePool:
    """The free pages of a cache, on the GPU: at first all of them, page 0 the first to go out."""

    def __init__(self, pages: int, device="cuda"):
        if pages <= 0:
            raise ValueError("pages must be positive")
        self.pages = pages
        self.stack = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.state = torch.tensor([pages, 0, 0, 0], dtype=torch.int32, device=device)
        self.device = self.stack.device
        self._c = _Pool(self.stack.data_ptr(), self.state.data_ptr(), pages)


def cache_bytes(num_layers: int, kv_heads: int, pages: int) -> int:
    return int(_load().tqp_cache_bytes(num_layers, kv_heads, pages))


def _pool_args(pool, table, seq_len):
    dev = pool.device
    _dev(table, "table", torch.int32, dev)
    if table.dim() != 2:
        raise ValueError("table must be [B][width]")
    B = table.shape[0]
    _dev(seq_len, "seq_len", torch.int32, dev, B)
    return dev, B


def assign(pool: PagePool, table, seq_len, new_tokens, rows: int, out=None):
    """Pages and slots for the new tokens of every sequence (tqp_assign): fills ``table`` [B][width], advances
    ``seq_len`` [B], and returns (slots int64 [rows], pos int32 [rows], row0 int32 [B+1], granted int32 [B]).
    ``rows``: the rows of the packed batch, at least the sum of new_tokens. ``out``: the four tensors to write to."""
    L = _load()
    dev, B = _pool_args(pool, table, seq_len)
    _dev(new_tokens, "new_tokens", torch.int32, dev, B)
    rows = int(rows)
    if out is None:
        out = (torch.empty(rows, dtype=torch.int64, device=dev), torch.empty(rows, dtype=torch.int32, device=dev),
               torch.empty(B + 1, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev))
    else:
        for name, t, dtype, n in zip(("slots", "pos", "row0", "granted"), out,
                                     (torch.int64, torch.int32, torch.int32, torch.int32), (rows, rows, B + 1, B)):
            _dev(t, name, dtype, dev, n)
    slots, pos, row0, granted = out
    with _on(dev) as stream:
        _check(L.tqp_assign(ctypes.byref(pool._c), table.data_ptr(), table.shape[1], B, seq_len.data_ptr(),
                            new_tokens.data_ptr(), rows, slots.data_ptr(), pos.data_ptr(), row0.data_ptr(),
                            granted.data_ptr(), stream))
    return slots, pos, row0, granted


def release(pool: PagePool, table, seq_len, keep) -> None:
    """Cuts every sequence to min(keep, seq_len) tokens and takes the pages it no longer needs back (tqp_release)."""
    L = _load()
    dev, B = _pool_args(pool, table, seq_len)
    _dev(keep, "keep", torch.int32, dev, B)
    with _on(dev) as stream:
        _check(L.tqp_release(ctypes.byref(pool._c), table.data_ptr(), table.shape[1], B, seq_len.data_ptr(),
                             keep.data_ptr(), stream))


def _cache_of(params: Params, cache: Cache):
    if cache.num_layers != params.num_layers or cache.kv_heads != params.kv_heads:
        raise ValueError("the cache has other layers or heads than params")
    return ctypes.byref(cache._c)


def append(params: Params, cache: Cache, k, v, slots, pos, layer0: int = 0) -> None:
    """Quantizes k, v [nlayers][rows][kv_heads][64] into the cache (tqp_append). ``slots`` int64 [rows] and ``pos``
    int32 [rows] come from assign(). k and v may be slices (strides in multiples of 8 elements)."""
    L = _load()
    dev = cache.device
    p, c = params.c(dev), _cache_of(params, cache)
    kr, vr = _rows(k, "k", params.io_dtype, params.kv_heads, dev), _rows(v, "v", params.io_dtype, params.kv_heads, dev)
    if k.shape != v.shape:
        raise ValueError("k and v must have the same shape")
    nl, rows = k.shape[:2]
    _dev(slots, "slots", torch.int64, dev, rows)
    _dev(pos, "pos", torch.int32, dev, rows)
    with _on(dev) as stream:
        _check(L.tqp_append(ctypes.byref(p), c, ctypes.byref(kr), ctypes.byref(vr), rows, layer0, nl,
                            slots.data_ptr(), pos.data_ptr(), stream))


def workspace_bytes(params: Params, nlayers: int, B: int, max_new: int, max_len: int) -> int:
    """Bytes of the workspace that attend() needs for these sizes (0 for most)."""
    return int(_load().tqp_workspace_bytes(ctypes.byref(params.c()), nlayers, B, max_new, max_len))


def attend(params: Params, cache: Cache, q, pos, row0, table, seq_len, max_new: int, max_len: int, causal: bool = True,
           layer0: int = 0, out=None, workspace=None) -> torch.Tensor:
    """Attention of the query rows q [nlayers][rows][num_heads][64] over the pages (tqp_attend): row t of sequence b
    sees the sequence's tokens j < seq_len[b], and with ``causal`` those up to its own position. ``max_new`` and
    ``max_len`` bound the rows and tokens of a sequence. ``workspace``: a tensor of workspace_bytes(...) bytes, zeroed
    before its first use (without one that is large enough a new one is made). Returns out
    [nlayers][rows][num_heads][64]."""
    L = _load()
    dev = cache.device
    p, c = params.c(dev), _cache_of(params, cache)
    qr = _rows(q, "q", params.io_dtype, params.num_heads, dev)
    nl, rows = q.shape[:2]
    _dev(table, "table", torch.int32, dev)
    if table.dim() != 2:
        raise ValueError("table must be [B][width]")
    B, width = table.shape
    _dev(pos, "pos", torch.int32, dev, rows)
    _dev(row0, "row0", torch.int32, dev, B + 1)
    _dev(seq_len, "seq_len", torch.int32, dev, B)
    dtype = torch.float32 if params.flags & OUT_FP32 else params.io_dtype
    if out is None:
        out = torch.empty(q.shape, dtype=dtype, device=dev)
    else:
        _dev(out, "out", dtype, dev)
        if out.shape != q.shape:
            raise ValueError("out must have the shape of q")
    max_new, max_len = int(max_new), int(max_len)
    pr = ctypes.byref(p)
    need = L.tqp_workspace_bytes(pr, nl, B, max_new, max_len)
    size = 0
    if need:
        if workspace is not None:
            if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or workspace.device != dev:
                raise TypeError("workspace must be a GPU tensor on the cache's device")
            if not workspace.is_contiguous():
                raise ValueError("workspace must be contiguous")
            size = workspace.numel() * workspace.element_size()
        if size < need:
            workspace, size = torch.zeros(need, dtype=torch.uint8, device=dev), need
    with _on(dev) as stream:
        _check(L.tqp_attend(pr, c, ctypes.byref(qr), rows, B, layer0, nl, pos.data_ptr(), row0.data_ptr(),
                            table.data_ptr(), width, seq_len.data_ptr(), max_new, max_len, int(bool(causal)),
                            out.data_ptr(), workspace.data_ptr() if need else None, size, stream))
    return out
