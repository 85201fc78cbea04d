"""Serving from a paged cache: the binding of include/stlite_paged.h.

    cache = PagedCache.alloc(n_layers, n_q_heads, n_kv_heads, n_seqs, max_len)
    compress(p, q_win, k, v, out, cache=cache)            # the kept rows, into pages
    step = NewTokens([0, 1, 2, ...])                       # one new token per sequence
    cache.seq_lens += 1                                    # lengths count the new tokens
    q = paged_append(cache, step, q, k, v, positions, rope)
    o = paged_attention(cache, step, q)

As in ``stlite``, every function only checks and marshals its arguments; all
arithmetic runs in the library's gfx950 kernels.  Tensors are bf16 or fp16, of
the pool's type and on its device.  Everything runs on ``stream`` (the device's
current one by default), allocates nothing where ``q_out``, ``out`` and
``workspace`` are given, and follows ``seq_lens`` and ``page_table`` on the
device, so that a step can be captured into a graph and replayed (the cache, the
batch and the call's tensors live as long as the graph).  With a
``torch.cuda.Stream`` the call's tensors, the batch's among them, may be dropped
at once; with the handle of a stream the caller keeps them until the work has run.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import numpy as np
import torch

from .stlite import _CPaged, _CRope, _CRows, _check, load

HEAD_DIM = 128
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


def _is(t, name, shape, dtype, device):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ' (not contiguous)'}")


class _On:
    """The device of a call, made current while it runs, and the handle of its stream."""

    def __init__(self, device, stream):
        if device.type != "cuda":
            raise ValueError(f"the cache is on {device}: the kernels run on a GPU")
        if stream is None:
            self.stream = torch.cuda.current_stream(device)
            self.handle, self.own = self.stream.cuda_stream, True
        else:
            at = getattr(stream, "device", device)  # (a handle does not know)
            if at != device:
                raise ValueError(f"the stream is on {at}, the cache on {device}")
            self.stream = stream
            self.handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
            self.own = self.handle == torch.cuda.current_stream(device).cuda_stream
        self.device, self.before = device, torch.cuda.current_device()
        if self.before != device.index:
            torch.cuda.set_device(device.index)

    def new(self, shape, dtype):
        """A tensor for this call's stream."""
        t = torch.empty(shape, dtype=dtype, device=self.device)
        if not self.own:
            s = self.stream if hasattr(self.stream, "cuda_stream") else torch.cuda.ExternalStream(self.handle, self.device)
            s.wait_stream(torch.cuda.current_stream(self.device))  # what used this memory before
            t.record_stream(s)
        return t

    def keep(self, *tensors):
        """The call's tensors: their memory is not given away before the stream has used it, should the caller drop them.
        (Not for a stream that the caller made, which may be gone when they are freed.)"""
        if type(self.stream) is torch.cuda.Stream:
            for t in tensors:
                if t is not None:
                    t.record_stream(self.stream)

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        if self.before != self.device.index:
            torch.cuda.set_device(self.before)


class _Fixed:
    """Attributes (``_fixed``) that the C structs took over at construction: set once, so that no call goes by another."""

    _fixed = ()

    def __setattr__(self, name, value):
        if name in self._fixed and self.__dict__.get(name, value) is not value:  # (``+=`` on a tensor assigns the same one)
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: make another {type(self).__name__}, or write into "
                                 "the tensor it holds")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{type(self).__name__}.{name} is fixed")
        super().__delattr__(name)


class Rope(_Fixed):
    """The position rotation (stlite_rope): one position axis, or three with ``sections`` pairs each."""

    _fixed = ("n_axes", "c")

    def __init__(self, theta: float = 1e6, sections=(64,), interleaved: bool = False):
        if len(sections) not in (1, 3) or sum(sections) != HEAD_DIM // 2 or min(sections) < 0:
            raise ValueError(f"sections must be (64,) or three counts that add up to 64, got {tuple(sections)}")
        self.n_axes = len(sections)
        self.c = _CRope(float(theta), int(bool(interleaved)), self.n_axes, (ctypes.c_int32 * 3)(*sections), 0)


class NewTokens(_Fixed):
    """The new tokens of a call: prefix sums over the sequences, on the host and the device, which stay the same."""

    _fixed = ("h", "d", "total", "_h", "_d")

    def __init__(self, cu_new, device="cuda"):
        given = np.asarray(cu_new)
        if given.ndim != 1 or len(given) < 2:
            raise ValueError("cu_new must be a list of n_seqs + 1 prefix sums")
        with np.errstate(invalid="ignore"):
            self.h = given.astype(np.int32)
        if not (self.h == given).all():
            raise ValueError("cu_new must hold whole numbers of 32 bits")
        self.h.setflags(write=False)
        self.d = torch.from_numpy(self.h.copy()).to(device)
        self.total = int(self.h[-1])
        self._h, self._d = self.h.ctypes.data, self.d.data_ptr()  # (a microsecond each time they are asked for)

    def __reduce__(self):  # a copy has addresses of its own
        return NewTokens, (self.h, self.d.device)


class PagedCache(_Fixed):
    """A pool of pages [n_layers][n_kv_heads][n_pages][page_size][128], the sequences' page table
    [n_seqs][max_pages] int32 and their lengths [n_seqs] int32.  ``max_len``: no sequence grows longer.

    The tensors are the cache's for good (a captured graph and the caches of single layers hold them too): other
    lengths or pages are written into them, ``cache.seq_lens.copy_(lens)``."""

    _fixed = ("k", "v", "page_table", "seq_lens", "tensors", "n_layers", "n_q_heads", "n_kv_heads", "n_pages", "page_size",
              "n_seqs", "max_pages", "max_len", "dtype", "device", "_c")

    def __init__(self, k, v, page_table, seq_lens, n_q_heads: int, max_len: Optional[int] = None):
        if k.dim() != 5 or k.shape[4] != HEAD_DIM or k.dtype not in _DTYPES:
            raise ValueError(f"k must be [n_layers, n_kv_heads, n_pages, page_size, {HEAD_DIM}] bf16 or fp16, got "
                             f"{k.dtype} {tuple(k.shape)}")
        if page_table.dim() != 2:
            raise ValueError("page_table must be [n_seqs, max_pages]")
        _is(k, "k", k.shape, k.dtype, k.device)
        _is(v, "v", k.shape, k.dtype, k.device)
        _is(page_table, "page_table", page_table.shape, torch.int32, k.device)
        _is(seq_lens, "seq_lens", page_table.shape[:1], torch.int32, k.device)
        self.k, self.v, self.page_table, self.seq_lens = self.tensors = k, v, page_table, seq_lens
        self.n_layers, self.n_kv_heads, self.n_pages, self.page_size = k.shape[:4]
        self.n_seqs, self.max_pages = page_table.shape
        self.n_q_heads, self.dtype, self.device = int(n_q_heads), k.dtype, k.device
        self.max_len = self.max_pages * self.page_size if max_len is None else int(max_len)
        for name in ("n_q_heads", "max_len", "n_pages", "max_pages", "n_seqs"):
            if not -2 ** 31 <= getattr(self, name) < 2 ** 31:  # (ctypes would cut it)
                raise ValueError(f"{name} {getattr(self, name)} does not fit in 32 bits")
        self._c = _CPaged(self.n_layers, self.n_q_heads, self.n_kv_heads, HEAD_DIM, _DTYPES[k.dtype], self.page_size,
                          self.n_pages, self.n_seqs, self.max_pages, self.max_len, 0, k.data_ptr(), v.data_ptr(),
                          page_table.data_ptr(), seq_lens.data_ptr(), None, None)

    def __reduce__(self):  # a copy has addresses of its own
        return PagedCache, (self.k, self.v, self.page_table, self.seq_lens, self.n_q_heads, self.max_len)

    @classmethod
    def alloc(cls, n_layers: int, n_q_heads: int, n_kv_heads: int, n_seqs: int, max_len: int, page_size: int = 64,
              dtype=torch.bfloat16, device="cuda"):
        """A zeroed pool with room for every sequence: sequence s owns the pages s * max_pages .. of it."""
        pages = -(-max_len // page_size)
        pool = [torch.zeros((n_layers, n_kv_heads, n_seqs * pages, page_size, HEAD_DIM), dtype=dtype, device=device)
                for _ in range(2)]
        table = torch.arange(n_seqs * pages, dtype=torch.int32, device=device).view(n_seqs, pages)
        return cls(*pool, table, torch.zeros(n_seqs, dtype=torch.int32, device=device), n_q_heads, max_len)

    def layer(self, i: int) -> "PagedCache":
        """Layer i alone, on the same pages and lengths: what a model's layer loop appends to and attends over."""
        if not 0 <= i < self.n_layers:
            raise ValueError(f"layer {i} of {self.n_layers}")
        return PagedCache(self.k[i:i + 1], self.v[i:i + 1], self.page_table, self.seq_lens, self.n_q_heads, self.max_len)

    def _struct(self, batch: Optional[NewTokens]):
        c = _CPaged.from_buffer_copy(self._c)
        if batch is not None:
            if len(batch.h) != self.n_seqs + 1:
                raise ValueError(f"the batch has {len(batch.h) - 1} sequences, the cache {self.n_seqs}")
            if batch.d.device != self.device:
                raise ValueError(f"the batch is on {batch.d.device}, the cache on {self.device}")
            c.total_new, c.cu_new, c.h_cu_new = batch.total, batch._d, batch._h
        return c

    def validate(self, batch: NewTokens, page_table=None, seq_lens=None) -> None:
        """stlite_paged_validate; page_table and seq_lens: the host's copies of what the device holds."""
        table = None if page_table is None else np.ascontiguousarray(page_table, dtype=np.int32)
        lens = None if seq_lens is None else np.ascontiguousarray(seq_lens, dtype=np.int32)
        if table is not None and table.shape != (self.n_seqs, self.max_pages):
            raise ValueError(f"page_table must be {(self.n_seqs, self.max_pages)}, got {table.shape}")
        if lens is not None and lens.shape != (self.n_seqs,):
            raise ValueError(f"seq_lens must be {(self.n_seqs,)}, got {lens.shape}")
        _check(load().stlite_paged_validate(ctypes.byref(self._struct(batch)),
                                            None if table is None else table.ctypes.data,
                                            None if lens is None else lens.ctypes.data), "stlite_paged_validate")

    def workspace_size(self, batch: NewTokens) -> int:
        n = ctypes.c_size_t(0)
        _check(load().stlite_paged_workspace_size(ctypes.byref(self._struct(batch)), ctypes.byref(n)),
               "stlite_paged_workspace_size")
        return n.value

    def workspace(self, batch: NewTokens):
        """Workspace of paged_attention for this batch.  Calls that share it must be ordered on one stream."""
        return torch.empty(max(self.workspace_size(batch), 256), dtype=torch.uint8, device=self.device)


def _rows(t, name, cache, batch, heads):
    n = batch.total
    if t.shape != (cache.n_layers, n, heads, HEAD_DIM) or t.dtype != cache.dtype or t.device != cache.device:
        raise ValueError(f"{name} must be {cache.dtype} {(cache.n_layers, n, heads, HEAD_DIM)} on {cache.device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    layer, token, head, dim = t.stride()
    if n and (dim != 1 or (head != HEAD_DIM and heads > 1)):
        raise ValueError(f"{name}: a token's heads must lie one after another (strides {t.stride()})")
    # (a size-1 axis may carry any stride)
    return _CRows(t.data_ptr(), token if n > 1 else heads * HEAD_DIM, layer if cache.n_layers > 1 else 0)


def _check_source(cache: PagedCache, p, k, v) -> None:
    """k and v of a compaction: rows of the pool's type, or 16-bit patterns as integers, which carry no type."""
    if p.d["cu_budget"].device != cache.device:
        raise ValueError(f"the problem is on {p.d['cu_budget'].device}, the cache on {cache.device}")
    n = cache.n_layers * cache.n_kv_heads * p.total_tokens * HEAD_DIM
    for t, name in ((k, "k"), (v, "v")):
        if (t.numel() != n or t.dtype not in (cache.dtype, torch.int16, torch.uint16) or not t.is_contiguous()
                or t.device != cache.device):
            raise ValueError(f"{name} must be a contiguous tensor of {n} {cache.dtype} elements (or their bits as 16-bit "
                             f"integers) on {cache.device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def check_compression(cache: PagedCache, p, k, v) -> None:
    """That the compression pass (problem p, bf16) can end in ``cache``; raises ValueError where it cannot."""
    if cache.dtype != torch.bfloat16:
        raise ValueError(f"the compression pass is bf16, the cache {cache.dtype}")
    for what, mine, its in (("layers", cache.n_layers, p.n_layers), ("kv heads", cache.n_kv_heads, p.n_kv_heads),
                            ("sequences", cache.n_seqs, p.n_seqs)):
        if mine != its:
            raise ValueError(f"the problem has {its} {what}, the cache {mine}")
    kept = int(np.diff(p.h["cu_budget"]).max())
    if kept > cache.max_len:
        raise ValueError(f"a sequence keeps {kept} rows, more than the cache's max_len = {cache.max_len}")
    _check_source(cache, p, k, v)


def paged_compact(cache: PagedCache, p, k, v, kept, per_layer: bool = False, stream=None) -> None:
    """The kept rows of the compression (problem p) into cache's pages; cache.seq_lens become the budgets."""
    _check_source(cache, p, k, v)
    lists = cache.n_layers if per_layer else cache.n_layers * cache.n_kv_heads
    if (kept.dtype != torch.int32 or not kept.is_contiguous() or kept.device != cache.device
            or (p.total_budget and kept.numel() != lists * p.total_budget)):
        raise ValueError(f"kept must be a contiguous int32 tensor of {lists} x {p.total_budget} on {cache.device}")
    with _On(cache.device, stream) as on:
        if not on.own:
            on.keep(k, v, kept, p.d["cu_budget"], *cache.tensors)
        _check(load().stlite_paged_compact(p.ref, ctypes.byref(cache._struct(None)), k.data_ptr(), v.data_ptr(),
                                           kept.data_ptr(), int(bool(per_layer)), on.handle), "stlite_paged_compact")


def paged_append(cache: PagedCache, batch: NewTokens, q, k, v, positions=None, rope: Optional[Rope] = None, q_norm=None,
                 k_norm=None, eps: float = 1e-6, q_out=None, stream=None):
    """Stores the new tokens' k (normed and rotated) and v in their pages; returns their q, normed and rotated.

    q, k, v: [n_layers, total_new, heads, 128], a token's heads one after another, any token and layer stride (slices
    of a fused projection); q may be None.  positions: int32 [axes, total_new]; q_norm, k_norm: [n_layers, 128]."""
    if (positions is None) != (rope is None):
        raise ValueError("positions and rope must be both given or both None")
    if positions is not None:
        _is(positions, "positions", (rope.n_axes, batch.total), torch.int32, cache.device)
    for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None:
            _is(t, name, (cache.n_layers, HEAD_DIM), cache.dtype, cache.device)
    rows = [_rows(k, "k", cache, batch, cache.n_kv_heads), _rows(v, "v", cache, batch, cache.n_kv_heads)]
    shape = (cache.n_layers, batch.total, cache.n_q_heads, HEAD_DIM)
    with _On(cache.device, stream) as on:
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
            rq = None
        else:
            rq = ctypes.byref(_rows(q, "q", cache, batch, cache.n_q_heads))
            if q_out is None:
                q_out = on.new(shape, cache.dtype)
            else:
                _is(q_out, "q_out", shape, cache.dtype, cache.device)
        if not on.own:
            on.keep(q, k, v, positions, q_norm, k_norm, q_out, batch.d, *cache.tensors)
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        _check(load().stlite_paged_append(ctypes.byref(cache._struct(batch)), None if rope is None else ctypes.byref(rope.c),
                                          ptr(positions), rq, ctypes.byref(rows[0]), ctypes.byref(rows[1]), ptr(q_norm),
                                          ptr(k_norm), float(eps), ptr(q_out), on.handle), "stlite_paged_append")
    return q_out


def paged_attention(cache: PagedCache, batch: NewTokens, q, out=None, workspace=None, scale: Optional[float] = None,
                    stream=None):
    """Causal attention of the new tokens' q [n_layers, total_new, n_q_heads, 128] over their sequences' pages, the new
    tokens themselves (appended before) among them.  scale: 1/sqrt(128) by default."""
    shape = (cache.n_layers, batch.total, cache.n_q_heads, HEAD_DIM)
    _is(q, "q", shape, cache.dtype, cache.device)
    if out is not None:
        _is(out, "out", shape, cache.dtype, cache.device)
    if workspace is not None and (workspace.device != cache.device or not workspace.is_contiguous()):
        raise ValueError(f"workspace must be contiguous and on {cache.device}")
    with _On(cache.device, stream) as on:
        if out is None:
            out = on.new(shape, cache.dtype)
        if workspace is None:
            workspace = on.new(max(cache.workspace_size(batch), 256), torch.uint8)
        if not on.own:
            on.keep(q, out, workspace, batch.d, *cache.tensors)
        _check(load().stlite_paged_attention(ctypes.byref(cache._struct(batch)), q.data_ptr(),
                                             1.0 / math.sqrt(HEAD_DIM) if scale is None else float(scale), out.data_ptr(),
                                             workspace.data_ptr(), workspace.numel() * workspace.element_size(), on.handle),
               "stlite_paged_attention")
    return out
