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
    room = torch.zeros(paged.workspace_bytes(params, 1, B, max_new, max_len), dtype=torch.uint8, device="cuda")
    slots, pos, row0, granted = paged.assign(pool, table, seq_len, new_tokens, rows)
    for l in range(L):                     # q, k, v: [1][rows][heads][64], rows of all sequences packed
        paged.append(params, cache, k, v, slots, pos, layer0=l)
        out = paged.attend(params, cache, q, pos, row0, table, seq_len, max_new, max_len, layer0=l, workspace=room)
    paged.release(pool, table, seq_len, keep)     # keep[b] = 0 where a sequence is finished

max_new and max_len are bounds that choose how attend runs: the closer they are
to the longest sequence's rows and tokens the better. Every call goes to the
current stream of its tensors' device, never synchronizes, and can be captured
into a graph.
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
_CAPACITY = -5
_COUNTERS = 16384                        # bytes at the start of a workspace that must be zero before its first use
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


def _fit(*numbers) -> None:
    """Raises unless all numbers are 32-bit ones (ctypes would cut them to that)."""
    if max(numbers) >= 2 ** 31 or min(numbers) < -2 ** 31:
        raise ValueError(f"{[n for n in numbers if not -2 ** 31 <= n < 2 ** 31]}: past 32 bits")


# A call's marshalling is a good part of a small launch's time (9 us of host work
# per append against 4 us of kernel, before): the checks of a call's tensors are
# one expression, and only where that fails do they run one by one, in order, to
# raise; structures that do not change are built with their object; the current
# stream comes as its raw handle.
def _dev(t, name: str, dtype, index: int | None = None, numel: int | None = None) -> torch.Tensor:
    """A contiguous tensor of the type, on GPU `index`, with at least `numel` elements."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{name} must be on GPU {index}, got {t.device}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} needs {numel} entries")
    return t


def _check_rows(t, name: str, dtype, nheads: int, index: int) -> None:
    """Raises unless t is a [nlayers][rows][heads][64] tensor of strides that the library takes."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 4 or t.shape[3] != 64 or t.shape[2] != nheads:
        raise ValueError(f"{name} must be [nlayers][rows][{nheads}][64]")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on GPU {index}, got {t.device}")
    if t.stride(3) != 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")


def _rows(t, shape) -> _Rows:
    s = t.stride()
    # (the stride of a dimension of one entry says nothing)
    return _Rows(t.data_ptr(), s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(index: int, f, *args) -> int:
    """f(*args, stream) with the tensors' GPU as the current one (the library launches there)."""
    if _current_device() == index:
        return f(*args, _raw_stream(index))
    with torch.cuda.device(index):
        return f(*args, _raw_stream(index))


@dataclass(frozen=True)
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

    def __post_init__(self):
        if self.io_dtype not in _IO:
            raise TypeError(f"io_dtype must be one of {[str(d) for d in _IO]}")
        cs = self.rope_cs
        if cs is not None:
            _dev(cs, "rope_cs", torch.float32)
            if cs.dim() != 3 or tuple(cs.shape[1:]) != (32, 2):
                raise ValueError("rope_cs must be [positions][32][2]")
        _fit(self.num_layers, self.num_heads, self.kv_heads, self.flags)
        c = _Params(64, self.num_layers, self.num_heads, self.kv_heads, _IO[self.io_dtype], self.flags,
                    self.softmax_scale, 0 if cs is None else cs.shape[0], None if cs is None else cs.data_ptr())
        object.__setattr__(self, "_c", c)
        object.__setattr__(self, "_index", None if cs is None else cs.get_device())
        object.__setattr__(self, "_out", torch.float32 if self.flags & OUT_FP32 else self.io_dtype)


class _Kept:
    """What the constructor sets stays, ``_c`` (the buffers' addresses) the last of it: the buffers' contents may change
    (``cache.scales *= 2``), the buffers may not."""

    _kept = frozenset()

    def __setattr__(self, name, value):
        if name in self._kept and value is not self.__dict__[name]:
            raise AttributeError(f"{name} of a {type(self).__name__} cannot be set: make another")
        object.__setattr__(self, name, value)
        if name == "_c":
            object.__setattr__(self, "_kept", frozenset(self.__dict__) | {"_kept"})

    def __delattr__(self, name):
        if name in self._kept:
            raise AttributeError(f"{name} of a {type(self).__name__} cannot be deleted: make another")
        object.__delattr__(self, name)


class Cache(_Kept):
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
                _dev(t, name, torch.float32 if last == 2 else torch.uint8, self.k_codes.get_device())
                if tuple(t.shape) != (*shape, last):
                    raise ValueError(f"{name} must be {[*shape, last]}")
        self.device, self._index = self.k_codes.device, self.k_codes.get_device()
        k = self.k_codes.view(torch.float8_e4m3fn).view(*shape, PAGE, 64)
        v = self.v_codes.view(torch.float8_e4m3fn).view(*shape, 4, 64, 4, 4).permute(0, 1, 2, 5, 3, 6, 4)
        self._values = (k, v, self.scales)
        self._c = _Cache(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.scales.data_ptr(), pages)

    def values(self):
        """Views of what the cache holds, as float8_e4m3fn tensors: keys [L][kv_heads][pages][64 tokens][64], values
        [L][kv_heads][pages][4][4][4][64] (token 16 i + 4 g + r at [i][g][r]), and the scales [L][kv_heads][pages][2]
        of keys and values that they are multiplied by."""
        return self._values


class PagePool(_Kept):
    """The free pages of a cache, on the GPU: at first all of them, page 0 the first to go out."""

    def __init__(self, pages: int, device="cuda"):
        if pages <= 0:
            raise ValueError("pages must be positive")
        self.pages = pages
        self.stack = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.state = torch.tensor([pages, 0, 0, 0], dtype=torch.int32, device=device)
        self.device, self._index = self.stack.device, self.stack.get_device()
        self._c = _Pool(self.stack.data_ptr(), self.state.data_ptr(), pages)


def cache_bytes(num_layers: int, kv_heads: int, pages: int) -> int:
    _fit(num_layers, kv_heads)
    return int(_load().tqp_cache_bytes(num_layers, kv_heads, pages))


def _pool_checks(pool: PagePool, table, seq_len, other, name: str) -> int:
    """The checks that assign and release share. Returns the number of sequences."""
    index, i32 = pool._index, torch.int32
    try:
        B = table.shape[0]
        fine = (table.dtype is i32 and seq_len.dtype is i32 and other.dtype is i32 and len(table.shape) == 2
                and table.is_contiguous() and seq_len.is_contiguous() and other.is_contiguous()
                and index >= 0 and table.get_device() == index and seq_len.get_device() == index
                and other.get_device() == index and seq_len.numel() >= B and other.numel() >= B)
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        _dev(table, "table", i32, index)
        if table.dim() != 2:
            raise ValueError("table must be [B][width]")
        B = table.shape[0]
        _dev(seq_len, "seq_len", i32, index, B)
        _dev(other, name, i32, index, B)
    return B


def assign(pool: PagePool, table, seq_len, new_tokens, rows: int, out=None):
    """Pages and slots for the new tokens of every sequence (tqp_assign): fills ``table`` [B][width], advances
    ``seq_len`` [B], and returns (slots int64 [rows], pos int32 [rows], row0 int32 [B+1], granted int32 [B]).
    ``rows``: the rows of the packed batch, at least the sum of new_tokens. ``out``: the four tensors to write to."""
    L = _lib or _load()
    B = _pool_checks(pool, table, seq_len, new_tokens, "new_tokens")
    rows = int(rows)
    _fit(rows, B, table.shape[1])
    if out is None:
        out = (torch.empty(rows, dtype=torch.int64, device=pool.device),
               *torch.empty(rows + B + 1 + B, dtype=torch.int32, device=pool.device).split_with_sizes((rows, B + 1, B)))
    else:
        for name, t, dtype, n in zip(("slots", "pos", "row0", "granted"), out,
                                     (torch.int64, torch.int32, torch.int32, torch.int32), (rows, rows, B + 1, B)):
            _dev(t, name, dtype, pool._index, n)
    slots, pos, row0, granted = out
    _check(_launch(pool._index, L.tqp_assign, ctypes.byref(pool._c), table.data_ptr(), table.shape[1], B,
                   seq_len.data_ptr(), new_tokens.data_ptr(), rows, slots.data_ptr(), pos.data_ptr(), row0.data_ptr(),
                   granted.data_ptr()))
    return slots, pos, row0, granted


def release(pool: PagePool, table, seq_len, keep) -> None:
    """Cuts every sequence to min(keep, seq_len) tokens and takes the pages it no longer needs back (tqp_release)."""
    L = _lib or _load()
    B = _pool_checks(pool, table, seq_len, keep, "keep")
    _fit(B, table.shape[1])
    _check(_launch(pool._index, L.tqp_release, ctypes.byref(pool._c), table.data_ptr(), table.shape[1], B,
                   seq_len.data_ptr(), keep.data_ptr()))


def _model_checks(params: Params, cache: Cache, kind=Cache) -> int:
    """The GPU of a call, once params and cache belong together. (A cache of another kind has other planes.)"""
    if type(cache) is not kind and not isinstance(cache, kind):
        raise TypeError(f"cache must be a {kind.__name__}")
    index = cache._index
    if cache.num_layers != params.num_layers or cache.kv_heads != params.kv_heads:
        raise ValueError("the cache has other layers or heads than params")
    if params._index is not None and params._index != index:
        raise ValueError("rope_cs must be on the cache's GPU")
    return index


def append(params: Params, cache: Cache, k, v, slots, pos=None, layer0: int = 0) -> None:
    """Quantizes k, v [nlayers][rows][kv_heads][64] into the cache (tqp_append). ``slots`` int64 [rows] and ``pos``
    int32 [rows] come from assign(); without rope_cs no ``pos`` is needed. k and v may be slices (strides in multiples
    of 8 elements)."""
    L = _lib or _load()
    index = _model_checks(params, cache)
    io, heads = params.io_dtype, params.kv_heads
    no_pos = pos is None and params.rope_cs is None
    try:
        shape = k.shape
        rows = shape[1]
        fine = (k.dtype is io and v.dtype is io and slots.dtype is torch.int64
                and len(shape) == 4 and shape[3] == 64 and shape[2] == heads and v.shape == shape
                and k.stride(3) == 1 and v.stride(3) == 1 and slots.is_contiguous()
                and index >= 0 and k.get_device() == index and v.get_device() == index
                and slots.get_device() == index and slots.numel() >= rows
                and (no_pos or (pos.dtype is torch.int32 and pos.is_contiguous() and pos.get_device() == index
                                and pos.numel() >= rows)))
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        _check_rows(k, "k", io, heads, index)
        _check_rows(v, "v", io, heads, index)
        if k.shape != v.shape:
            raise ValueError("k and v must have the same shape")
        _dev(slots, "slots", torch.int64, index, rows)
        if not no_pos:
            _dev(pos, "pos", torch.int32, index, rows)
    _fit(rows, layer0, shape[0])
    _check(_launch(index, L.tqp_append, ctypes.byref(params._c), ctypes.byref(cache._c), ctypes.byref(_rows(k, shape)),
                   ctypes.byref(_rows(v, shape)), rows, layer0, shape[0], slots.data_ptr(),
                   None if no_pos else pos.data_ptr()))


def workspace_bytes(params: Params, nlayers: int, B: int, max_new: int, max_len: int) -> int:
    """Bytes of the workspace that attend() needs for these sizes (0 for most)."""
    _fit(nlayers, B, max_new, max_len)
    return int(_load().tqp_workspace_bytes(ctypes.byref(params._c), nlayers, B, max_new, max_len))


def attend(params: Params, cache: Cache, q, pos, row0, table, seq_len, max_new: int, max_len: int, causal: bool = True,
           layer0: int = 0, out=None, workspace=None) -> torch.Tensor:
    """Attention of the query rows q [nlayers][rows][num_heads][64] over the pages (tqp_attend): row t of sequence b
    sees the sequence's tokens j < seq_len[b], and with ``causal`` those up to its own position. ``max_new`` and
    ``max_len`` bound the rows and tokens of a sequence. ``workspace``: a tensor of workspace_bytes(...) bytes whose
    first 16384 are zero before its first use (without one that is large enough every call makes a new one). Returns
    out [nlayers][rows][num_heads][64]."""
    L = _lib or _load()
    index = _model_checks(params, cache)
    io, heads, i32, dtype = params.io_dtype, params.num_heads, torch.int32, params._out
    try:
        shape = q.shape
        rows, B = shape[1], table.shape[0]
        fine = (q.dtype is io and len(shape) == 4 and shape[3] == 64 and shape[2] == heads and q.stride(3) == 1
                and pos.dtype is i32 and row0.dtype is i32 and table.dtype is i32 and seq_len.dtype is i32
                and len(table.shape) == 2 and pos.is_contiguous() and row0.is_contiguous() and table.is_contiguous()
                and seq_len.is_contiguous() and index >= 0 and q.get_device() == index and pos.get_device() == index
                and row0.get_device() == index and table.get_device() == index and seq_len.get_device() == index
                and pos.numel() >= rows and row0.numel() > B and seq_len.numel() >= B)
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        _check_rows(q, "q", io, heads, index)
        _dev(table, "table", i32, index)
        if table.dim() != 2:
            raise ValueError("table must be [B][width]")
        _dev(pos, "pos", i32, index, q.shape[1])
        _dev(row0, "row0", i32, index, table.shape[0] + 1)
        _dev(seq_len, "seq_len", i32, index, table.shape[0])
    max_new, max_len = int(max_new), int(max_len)
    _fit(rows, B, table.shape[1], layer0, shape[0], max_new, max_len)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=cache.device)
    else:
        _dev(out, "out", dtype, index)
        if out.shape != shape:
            raise ValueError("out must have the shape of q")
    size = 0
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or index < 0:
            raise TypeError("workspace must be a GPU tensor on the cache's device")
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        size = workspace.numel() * workspace.element_size()
    args = (ctypes.byref(params._c), ctypes.byref(cache._c), ctypes.byref(_rows(q, shape)), rows, B, layer0, shape[0],
            pos.data_ptr(), row0.data_ptr(), table.data_ptr(), table.shape[1], seq_len.data_ptr(), max_new,
            max_len, 1 if causal else 0, out.data_ptr())
    status = _launch(index, L.tqp_attend, *args, None if workspace is None else workspace.data_ptr(), size)
    if status == _CAPACITY:              # (refused before anything was launched)
        need = L.tqp_workspace_bytes(args[0], shape[0], B, max_new, max_len)
        if need > size:
            workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
            workspace[:_COUNTERS].zero_()
            status = _launch(index, L.tqp_attend, *args, workspace.data_ptr(), need)
    _check(status)
    return out
