"""A serving step around a paged 4-bit KV cache for MI355X: norm and rotation of queries and keys, the append that
quantizes keys and values, reading them back, attention over them, and the verification of drafted tokens.

Thin ctypes binding of ``libturboesm_serve.so`` (C ABI in ``include/turboesm_serve.h``). Pages, slots and row offsets
are those of the ``paged`` module (``PagePool``, ``assign``, ``release``), and so is ``Params``. Beside ``paged.Cache``
the cache here holds e2m1 codes with a power-of-two scale per token and head, in the Hadamard basis: 66 bytes per
cached token and key/value head, where that takes 128. Types are fp16, bf16 and fp32. If the library is not built,
calls raise ``RuntimeError``.

A step with drafted tokens, where a model norms its queries and keys:

    pool, cache = paged.PagePool(pages), serve.Cache4(L, kv_heads, pages)
    before = paged.Params(L, heads, kv_heads, rope_cs, io_dtype=torch.bfloat16)     # turns q and k
    params = paged.Params(L, heads, kv_heads, io_dtype=torch.bfloat16)              # takes them as they are then
    room = torch.zeros(max(serve.workspace_bytes(params, 1, B, max_new, max_len), serve.verify_workspace_bytes(vocab, B)),
                       dtype=torch.uint8, device="cuda")
    slots, pos, row0, granted = paged.assign(pool, table, seq_len, new_tokens, rows)   # the last token and its drafts
    for l in range(L):                     # q, k, v: [1][rows][heads][64], slices of one projection's output
        q, k = serve.norm_rope(before, q, k, pos, q_weight[l:l + 1], k_weight[l:l + 1])
        serve.append(params, cache, k, v, slots, layer0=l)
        out = serve.attend(params, cache, q, pos, row0, table, seq_len, max_new, max_len, layer0=l, workspace=room)
    accepted, token, keep = serve.verify(target, draft, tokens, row0, uniform, uniform_next, seq_len, workspace=room)
    paged.release(pool, table, seq_len, keep)

Without drafts, or without such norms, the calls in question are left out; append and attend rotate k and q themselves
where their params have a table. Every call goes to the current stream of its tensors' device, never synchronizes, and
can be captured into a graph.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

from . import TQError
from .paged import _CAPACITY, _COUNTERS, _IO, MAX_SEQS, PAGE, Params, _check_rows, _dev, _fit, _Kept, _launch, _model_checks

__all__ = ["Cache4", "norm_rope", "append", "read", "attend", "verify", "workspace_bytes", "verify_workspace_bytes",
           "cache_bytes", "last_error", "lib_path", "MAX_AXES", "MAX_SEQS", "PAGE", "Params"]

MAX_AXES = 4

lib_path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libturboesm_serve.so")


class _Cache4(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("pages", ctypes.c_int64)]


_lib = None


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(lib_path):
        raise RuntimeError(f"{lib_path} is not built; run __graft_entry__.build() "
                           "or python -m paper_2603_26110_amd.build")
    L = ctypes.CDLL(lib_path)
    P, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    L.tqs_last_error.restype = ctypes.c_char_p
    L.tqs_cache_bytes.argtypes = [i32, i32, i64]
    L.tqs_cache_bytes.restype = i64
    L.tqs_norm_rope.argtypes = [P, P, P, i32, i32, P, P, f32, P, i32, P, P, P, P]
    L.tqs_norm_rope.restype = i32
    L.tqs_append.argtypes = [P, P, P, P, i32, i32, i32, P, P, P]
    L.tqs_append.restype = i32
    L.tqs_read.argtypes = [P, P, P, i32, i32, i32, P, P, P]
    L.tqs_read.restype = i32
    L.tqs_attend.argtypes = [P, P, P, i32, i32, i32, i32, P, P, P, i32, P, i32, i32, i32, P, P, sz, P]
    L.tqs_attend.restype = i32
    L.tqs_workspace_bytes.argtypes = [P, i32, i32, i32, i32]
    L.tqs_workspace_bytes.restype = sz
    L.tqs_verify.argtypes = [P, i64, P, i64, i32, i32, i32, i32, P, P, P, P, P, P, P, P, P, sz, P]
    L.tqs_verify.restype = i32
    L.tqs_verify_workspace_bytes.argtypes = [i32, i32]
    L.tqs_verify_workspace_bytes.restype = sz
    _lib = L
    return L


def last_error() -> str:
    return _load().tqs_last_error().decode()


def _check(status: int) -> None:
    if status != 0:
        raise TQError(f"status {status}: {last_error()}")


class Cache4(_Kept):
    """Pages in device memory: per (layer, key/value head, page) 2048 bytes of key codes, 2048 of value codes and 128
    scales. ``buffers``: the caller's own (k_codes, v_codes, scales), uint8, in place of new ones that hold zeros."""

    def __init__(self, num_layers: int, kv_heads: int, pages: int, device="cuda", buffers=None):
        if num_layers <= 0 or kv_heads <= 0 or pages <= 0:
            raise ValueError("num_layers, kv_heads and pages must be positive")
        self.num_layers, self.kv_heads, self.pages = num_layers, kv_heads, pages
        shape = (num_layers, kv_heads, pages)
        if buffers is None:
            self.k_codes = torch.zeros((*shape, PAGE * 32), dtype=torch.uint8, device=device)
            self.v_codes = torch.zeros((*shape, PAGE * 32), dtype=torch.uint8, device=device)
            self.scales = torch.full((*shape, 2 * PAGE), 127, dtype=torch.uint8, device=device)
        else:
            self.k_codes, self.v_codes, self.scales = buffers
            for name, t, last in (("k_codes", self.k_codes, PAGE * 32), ("v_codes", self.v_codes, PAGE * 32),
                                  ("scales", self.scales, 2 * PAGE)):
                _dev(t, name, torch.uint8, self.k_codes.get_device())
                if tuple(t.shape) != (*shape, last):
                    raise ValueError(f"{name} must be {[*shape, last]}")
        self.device, self._index = self.k_codes.device, self.k_codes.get_device()
        self._c = _Cache4(self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.scales.data_ptr(), pages)


def cache_bytes(num_layers: int, kv_heads: int, pages: int) -> int:
    _fit(num_layers, kv_heads)
    return int(_load().tqs_cache_bytes(num_layers, kv_heads, pages))


# As in the paged binding, the checks of a call's tensors are one expression, and only where that fails do they run one by
# one, in order, to raise. Rows go to the library as the bytes of their structure (norm_rope hands over four of them).
_pack_rows = struct.Struct("Pqqq").pack


def _rows(t, shape) -> bytes:
    s = t.stride()
    # (the stride of a dimension of one entry says nothing)
    return _pack_rows(t.data_ptr(), s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0)


def norm_rope(params: Params, q, k, pos=None, q_weight=None, k_weight=None, eps: float = 1e-6, sections=None, out=None):
    """Norms every head of q [nlayers][rows][num_heads][64] and k [nlayers][rows][kv_heads][64] (divided by the root of
    the mean of its squares and eps, times ``q_weight`` or ``k_weight``, fp32 [nlayers][64] or None for ones) and
    rotates it by its row's position (tqs_norm_rope). ``pos``: int32 [rows], or [axes][rows] with ``sections``, the
    pairs that each axis turns (32 in all). Without rope_cs nothing is rotated. Returns (q', k'), contiguous, or written to
    ``out``, two tensors of those shapes with strides in multiples of 8 elements: q and k themselves, say. What comes
    next takes params without a table."""
    L = _lib or _load()
    io, heads, kv_heads = params.io_dtype, params.num_heads, params.kv_heads
    turned = params.rope_cs is not None
    try:
        shape, kshape, index = q.shape, k.shape, q.get_device()
        nlayers, rows = shape[0], shape[1]
        fine = (q.dtype is io and k.dtype is io and index >= 0 and k.get_device() == index and len(shape) == 4
                and len(kshape) == 4 and shape[2] == heads and kshape[2] == kv_heads and shape[3] == 64 and kshape[3] == 64
                and kshape[0] == nlayers and kshape[1] == rows and q.stride(3) == 1 and k.stride(3) == 1
                and (q_weight is None or (q_weight.dtype is torch.float32 and q_weight.shape == (nlayers, 64)
                                          and q_weight.is_contiguous() and q_weight.get_device() == index))
                and (k_weight is None or (k_weight.dtype is torch.float32 and k_weight.shape == (nlayers, 64)
                                          and k_weight.is_contiguous() and k_weight.get_device() == index))
                and (not turned or (params._index == index and pos.dtype is torch.int32 and pos.is_contiguous()
                                    and pos.get_device() == index and 1 <= len(pos.shape) <= 2 and pos.shape[-1] == rows)))
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        if not isinstance(q, torch.Tensor) or not q.is_cuda:
            raise TypeError("q must be a GPU tensor")
        index = q.get_device()
        _check_rows(q, "q", io, heads, index)
        _check_rows(k, "k", io, kv_heads, index)
        if q.shape[:2] != k.shape[:2]:
            raise ValueError("q and k must have the same layers and rows")
        for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
            if w is not None:
                _dev(w, name, torch.float32, index)
                if tuple(w.shape) != (q.shape[0], 64):
                    raise ValueError(f"{name} must be [{q.shape[0]}][64]")
        if turned:
            if params._index != index:
                raise ValueError("rope_cs must be on the GPU of q")
            _dev(pos, "pos", torch.int32, index)
            raise ValueError("pos must be [rows] or [axes][rows]")
    axes, parts = 1, None
    if turned:
        axes = pos.shape[0] if len(pos.shape) == 2 else 1
        if sections is not None:
            sections = [int(n) for n in sections]
            if len(sections) != axes:
                raise ValueError("sections must have an entry for each axis of pos")
            _fit(0, *sections)
            parts = struct.pack(f"{axes}i", *sections)
        elif axes != 1:
            raise ValueError("several axes need sections")
    if out is None:
        q_out, k_out = torch.empty(shape, dtype=io, device=q.device), torch.empty(kshape, dtype=io, device=q.device)
    else:
        q_out, k_out = out
        for name, t, x in (("q out", q_out, q), ("k out", k_out, k)):
            _check_rows(t, name, io, x.shape[2], index)
            if t.shape != x.shape:
                raise ValueError(f"{name} must have the shape of its input")
    _fit(rows, nlayers)
    _check(_launch(index, L.tqs_norm_rope, ctypes.byref(params._c), _rows(q, shape), _rows(k, kshape), rows, nlayers,
                   None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
                   eps, pos.data_ptr() if turned else None, axes, parts, _rows(q_out, shape), _rows(k_out, kshape)))
    return q_out, k_out


def append(params: Params, cache: Cache4, k, v, slots, pos=None, layer0: int = 0) -> None:
    """Quantizes k, v [nlayers][rows][kv_heads][64] into the cache (tqs_append). ``slots`` int64 [rows] and ``pos``
    int32 [rows] come from paged.assign(); without rope_cs no ``pos`` is needed. k and v may be slices (strides in
    multiples of 8 elements)."""
    L = _lib or _load()
    index = _model_checks(params, cache, Cache4)
    io, heads, turned = params.io_dtype, params.kv_heads, params.rope_cs is not None
    try:
        shape = k.shape
        rows = shape[1]
        fine = (k.dtype is io and v.dtype is io and slots.dtype is torch.int64 and len(shape) == 4 and shape[3] == 64
                and shape[2] == heads and v.shape == shape and k.stride(3) == 1 and v.stride(3) == 1
                and slots.is_contiguous() and index >= 0 and k.get_device() == index and v.get_device() == index
                and slots.get_device() == index and slots.numel() >= rows
                and (not turned or (pos.dtype is torch.int32 and pos.is_contiguous() and pos.get_device() == index
                                    and pos.numel() >= rows)))
    except (AttributeError, IndexError):
        fine = False
    if not fine:
        _check_rows(k, "k", io, heads, index)
        _check_rows(v, "v", io, heads, index)
        if k.shape != v.shape:
            raise ValueError("k and v must have the same shape")
        _dev(slots, "slots", torch.int64, index, rows)
        _dev(pos, "pos", torch.int32, index, rows)
    _fit(rows, layer0, shape[0])
    _check(_launch(index, L.tqs_append, ctypes.byref(params._c), ctypes.byref(cache._c), _rows(k, shape), _rows(v, shape),
                   rows, layer0, shape[0], slots.data_ptr(), pos.data_ptr() if turned else None))


def read(params: Params, cache: Cache4, slots, layer0: int = 0, nlayers: int | None = None, out=None):
    """What the cache holds in ``slots`` (int64 [rows]), for all layers from ``layer0`` on or the next ``nlayers``
    (tqs_read): (k, v), each [nlayers][rows][kv_heads][64] of the params' output type. Keys come rotated, as they were
    quantized. ``out``: the two tensors to write to."""
    L = _lib or _load()
    index = _model_checks(params, cache, Cache4)
    _dev(slots, "slots", torch.int64, index)
    rows = slots.numel()
    if nlayers is None:
        nlayers = max(params.num_layers - layer0, 0)
    _fit(rows, layer0, nlayers)
    shape = (max(nlayers, 0), rows, params.kv_heads, 64)
    if out is None:
        out = tuple(torch.empty(shape, dtype=params._out, device=cache.device) for _ in range(2))
    else:
        for name, t in zip(("k out", "v out"), out):
            _dev(t, name, params._out, index)
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must be {list(shape)}")
    k, v = out
    _check(_launch(index, L.tqs_read, ctypes.byref(params._c), ctypes.byref(cache._c), slots.data_ptr(), rows, layer0,
                   nlayers, k.data_ptr(), v.data_ptr()))
    return k, v


def workspace_bytes(params: Params, nlayers: int, B: int, max_new: int, max_len: int) -> int:
    """Bytes of the workspace that attend() needs for these sizes (0 for most)."""
    _fit(nlayers, B, max_new, max_len)
    return int(_load().tqs_workspace_bytes(ctypes.byref(params._c), nlayers, B, max_new, max_len))


def verify_workspace_bytes(vocab: int, B: int) -> int:
    """Bytes of the workspace that verify() needs for these sizes (0 for small vocabularies)."""
    _fit(vocab, B)
    return int(_load().tqs_verify_workspace_bytes(vocab, B))


def _workspace(workspace, index: int):
    """(address, bytes) of a caller's workspace, or (None, 0)."""
    if workspace is None:
        return None, 0
    if not isinstance(workspace, torch.Tensor) or workspace.get_device() != index or index < 0:
        raise TypeError("workspace must be a GPU tensor on the device of the call")
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _room(need: int, device) -> torch.Tensor:
    """A new workspace."""
    workspace = torch.empty(need, dtype=torch.uint8, device=device)
    workspace[:_COUNTERS].zero_()
    return workspace


def attend(params: Params, cache: Cache4, q, pos, row0, table, seq_len, max_new: int, max_len: int, causal: bool = True,
           layer0: int = 0, out=None, workspace=None) -> torch.Tensor:
    """Attention of the query rows q [nlayers][rows][num_heads][64] over the pages (tqs_attend): row t of sequence b
    sees the sequence's tokens j < seq_len[b], and with ``causal`` those up to its own position. ``max_new`` and
    ``max_len`` bound the rows and tokens of a sequence. ``workspace``: a tensor of workspace_bytes(...) bytes whose
    first 16384 are zero before its first use (without one that is large enough every call makes a new one). Returns
    out [nlayers][rows][num_heads][64]."""
    L = _lib or _load()
    index = _model_checks(params, cache, Cache4)
    io, heads, i32 = params.io_dtype, params.num_heads, torch.int32
    try:
        shape = q.shape
        rows, (B, width) = shape[1], table.shape
        fine = (q.dtype is io and len(shape) == 4 and shape[3] == 64 and shape[2] == heads and q.stride(3) == 1
                and pos.dtype is i32 and row0.dtype is i32 and table.dtype is i32 and seq_len.dtype is i32
                and pos.is_contiguous() and row0.is_contiguous() and table.is_contiguous()
                and seq_len.is_contiguous() and index >= 0 and q.get_device() == index and pos.get_device() == index
                and row0.get_device() == index and table.get_device() == index and seq_len.get_device() == index
                and pos.numel() >= rows and row0.numel() > B and seq_len.numel() >= B)
    except (AttributeError, IndexError, ValueError):
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
    _fit(rows, B, width, layer0, shape[0], max_new, max_len)
    if out is None:
        out = torch.empty(shape, dtype=params._out, device=cache.device)
    else:
        _dev(out, "out", params._out, index)
        if out.shape != shape:
            raise ValueError("out must have the shape of q")
    at, size = _workspace(workspace, index)
    args = (ctypes.byref(params._c), ctypes.byref(cache._c), _rows(q, shape), rows, B, layer0, shape[0],
            pos.data_ptr(), row0.data_ptr(), table.data_ptr(), width, seq_len.data_ptr(), max_new, max_len,
            1 if causal else 0, out.data_ptr())
    status = _launch(index, L.tqs_attend, *args, at, size)
    if status == _CAPACITY:              # (refused before anything was launched)
        need = L.tqs_workspace_bytes(args[0], shape[0], B, max_new, max_len)
        if need > size:
            workspace = _room(need, cache.device)
            status = _launch(index, L.tqs_attend, *args, workspace.data_ptr(), need)
    _check(status)
    return out


def _check_probabilities(t, name: str, dtype, shape, index: int) -> None:
    """Raises unless t is a [rows][vocab] tensor of strides that the library takes."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    if t.get_device() != index:
        raise ValueError(f"{name} must be on GPU {index}, got {t.device}")
    if shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the probabilities of a row must be contiguous")


def verify(target, draft, tokens, row0, uniform, uniform_next, seq_len=None, workspace=None):
    """Accepts or rejects drafted tokens and draws every sequence's next one (tqs_verify). Rows row0[b] .. row0[b+1]-1
    are a sequence's last token and its drafts: ``tokens`` int64 [rows]; ``target`` and ``draft`` [rows][vocab] (fp32,
    fp16 or bf16, rows at any stride) the probabilities of the token after each row by either model; ``draft`` None
    where drafts were not drawn but given. ``uniform`` fp32 [rows] and ``uniform_next`` fp32 [B]: random numbers in
    [0, 1). Returns (accepted int32 [B], next token int64 [B], keep int32 [B]); keep is what paged.release() takes where
    ``seq_len`` int32 [B] counts the rows in, and None without it. ``workspace``: as attend()'s, of
    verify_workspace_bytes(...) bytes."""
    L = _lib or _load()
    i32, f32 = torch.int32, torch.float32
    try:
        index, dtype, shape = target.get_device(), target.dtype, target.shape
        rows, vocab = shape
        B = row0.numel() - 1
        fine = (index >= 0 and dtype in _IO and (vocab == 1 or target.stride(1) == 1)
                and (draft is None or (draft.dtype is dtype and draft.shape == shape and draft.get_device() == index
                                       and (vocab == 1 or draft.stride(1) == 1)))
                and tokens.dtype is torch.int64 and row0.dtype is i32 and uniform.dtype is f32 and uniform_next.dtype is f32
                and tokens.is_contiguous() and row0.is_contiguous() and uniform.is_contiguous()
                and uniform_next.is_contiguous() and tokens.get_device() == index and row0.get_device() == index
                and uniform.get_device() == index and uniform_next.get_device() == index and tokens.numel() >= rows
                and B >= 0 and uniform.numel() >= rows and uniform_next.numel() >= B
                and (seq_len is None or (seq_len.dtype is i32 and seq_len.is_contiguous()
                                         and seq_len.get_device() == index and seq_len.numel() >= B)))
    except (AttributeError, ValueError):
        fine = False
    if not fine:
        if not isinstance(target, torch.Tensor) or not target.is_cuda:
            raise TypeError("target must be a GPU tensor")
        if target.dtype not in _IO:
            raise TypeError(f"target must be one of {[str(d) for d in _IO]}")
        if target.dim() != 2:
            raise ValueError("target must be [rows][vocab]")
        _check_probabilities(target, "target", target.dtype, target.shape, target.get_device())
        if draft is not None:
            _check_probabilities(draft, "draft", target.dtype, target.shape, target.get_device())
        index, rows = target.get_device(), target.shape[0]
        _dev(row0, "row0", i32, index, 1)
        _dev(tokens, "tokens", torch.int64, index, rows)
        _dev(uniform, "uniform", f32, index, rows)
        _dev(uniform_next, "uniform_next", f32, index, row0.numel() - 1)
        _dev(seq_len, "seq_len", i32, index, row0.numel() - 1)
    _fit(rows, vocab, B)
    at, size = _workspace(workspace, index)
    device = target.device
    out = torch.empty((2, B), dtype=i32, device=device)
    accepted, keep = out[0], out[1]
    token = torch.empty(B, dtype=torch.int64, device=device)
    strides = [t.stride(0) if t is not None and rows > 1 else vocab for t in (target, draft)]
    args = (target.data_ptr(), strides[0], None if draft is None else draft.data_ptr(), strides[1], _IO[dtype], vocab,
            rows, B, tokens.data_ptr(), row0.data_ptr(), uniform.data_ptr(), uniform_next.data_ptr(),
            None if seq_len is None else seq_len.data_ptr(), accepted.data_ptr(), token.data_ptr(),
            None if seq_len is None else keep.data_ptr())
    status = _launch(index, L.tqs_verify, *args, at, size)
    if status == _CAPACITY:              # (refused before anything was launched)
        need = L.tqs_verify_workspace_bytes(vocab, B)
        if need > size:
            workspace = _room(need, device)
            status = _launch(index, L.tqs_verify, *args, workspace.data_ptr(), need)
    _check(status)
    return accepted, token, None if seq_len is None else keep
