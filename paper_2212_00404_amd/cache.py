"""Binding of the cache of keys and values in pages: ``Cache`` (the pool),
``cache_write``, ``cache_read`` and ``attend_cache`` (attention of new tokens over
what it holds).

Argument marshalling only, as in ``tokens.py``; ``include/dconv.h`` has the
definitions.  Nothing here is recorded by autograd.
"""
from __future__ import annotations

import math
import struct

import torch

from .dconv import _call, _check, load
from .tokens import _DTYPES, _pack, _plain, _ptr, _shaped, _tensor, _workspace

_PLAIN, _E4M3, _E2M1 = 0, 1, 2
_FORMATS = {"e4m3": _E4M3, "e2m1": _E2M1}
_STORED = {torch.float8_e4m3fn: _E4M3, torch.uint8: _E2M1}
_SCALE = torch.float8_e8m0fnu

# The C structs of include/dconv.h.
_CACHE = struct.Struct("@6i12q")
_ROWS = struct.Struct("@4i5q")
_ATTEND = struct.Struct("@9if5q")


class Cache:
    """A pool of pages of keys and values.

    ``k``, ``v``: ``[pages, page_size, heads, D]``, any strides with a contiguous
    last dimension, of fp32, fp16 or bf16; or ``float8_e4m3fn``; or ``uint8`` for
    two elements of 4 bits (sign, 2 bits of exponent, 1 of mantissa) in a byte,
    ``[..., D / 2]``, the first in the low half.  The latter two stand for code *
    scale, with ``k_scale``, ``v_scale`` ``[pages, page_size, heads, D / 32]`` of
    ``float8_e8m0fnu``: a power of two for each 32 neighbours of a head.

    ``new`` allocates one whose pages hold the tokens of one head after another.
    """
    __slots__ = ("k", "v", "k_scale", "v_scale", "pages", "page_size", "heads", "dim", "format", "dtype",
                 "device", "index", "_shape")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None):
        if not isinstance(k, torch.Tensor):
            raise ValueError("k must be a torch.Tensor")
        self.format = _STORED.get(k.dtype, _PLAIN)
        if self.format == _PLAIN and k.dtype not in _DTYPES:
            raise ValueError("k must be float32, float16, bfloat16, float8_e4m3fn or uint8 (two elements of "
                             "4 bits), got %s" % k.dtype)
        _tensor(k, "k", 4, k.dtype)
        _tensor(v, "v", 4, k.dtype, k.device)
        _shaped(v, "v", k.shape)
        self.pages, self.page_size, self.heads, last = k.shape
        self.dim = last * 2 if self.format == _E2M1 else last
        self.dtype = None if self.format else k.dtype
        if min(k.shape) < 1:
            raise ValueError("a cache has a page, a slot, a head and an element: k is %r" % (tuple(k.shape),))
        if self.format:
            if self.dim % 32:
                raise ValueError("heads of a cache of 8 or 4 bits are a multiple of 32, got %d" % self.dim)
            for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
                _tensor(t, name, 4, _SCALE, k.device)
                _shaped(t, name, (*k.shape[:3], self.dim // 32))
        elif k_scale is not None or v_scale is not None:
            raise ValueError("a cache of %s has no scales" % k.dtype)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.index = k.device, k.get_device()
        none = (0, 0, 0)
        self._shape = _pack(_CACHE, self.pages, self.page_size, self.heads, self.dim, self.format,
                            _DTYPES.get(k.dtype, 0), *k.stride()[:3], *v.stride()[:3],
                            *(k_scale.stride()[:3] if self.format else none),
                            *(v_scale.stride()[:3] if self.format else none))

    @classmethod
    def new(cls, pages: int, page_size: int, heads: int, dim: int, kind=torch.bfloat16, device="cuda") -> "Cache":
        """``kind``: fp32, fp16 or bf16, or ``"e4m3"`` or ``"e2m1"``."""
        if kind in _FORMATS and dim % 32:
            raise ValueError("heads of a cache of 8 or 4 bits are a multiple of 32, got %d" % dim)
        store = {"e4m3": torch.float8_e4m3fn, "e2m1": torch.uint8}.get(kind, kind)
        if store not in _DTYPES and kind not in _FORMATS:
            raise ValueError("kind must be a type of %s or one of %s, got %r"
                             % (sorted(map(str, _DTYPES)), sorted(_FORMATS), kind))

        def pool(last, dtype):
            return torch.empty((pages, heads, page_size, last), dtype=dtype, device=device).transpose(1, 2)

        last = dim // 2 if kind == "e2m1" else dim
        scales = [pool(dim // 32, torch.uint8).view(_SCALE) for _ in range(2)] if kind in _FORMATS else [None, None]
        return cls(pool(last, store), pool(last, store), *scales)

    def _pointers(self):
        return self.k.data_ptr(), self.v.data_ptr(), _ptr(self.k_scale), _ptr(self.v_scale)


def _batch(cache, table, lengths, offsets, N):
    """Checks of what names the rows' places; (sequences, width of the table, its
    stride)."""
    if not isinstance(cache, Cache):
        raise ValueError("cache must be a Cache")
    dev, index = cache.device, cache.index
    if not _plain(table, 2, torch.int32, index):
        _tensor(table, "table", 2, torch.int32, dev)
    B, width = table.shape
    if not (_plain(lengths, 1, torch.int32, index) and lengths.shape[0] == B):
        _tensor(lengths, "lengths", 1, torch.int32, dev)
        _shaped(lengths, "lengths", (B,))
    if offsets is None:
        if N % B if B else N:
            raise ValueError("%d rows are not as many for each of %d sequences: pass offsets" % (N, B))
    elif not (_plain(offsets, 1, torch.int32, index) and offsets.shape[0] == B + 1):
        _tensor(offsets, "offsets", 1, torch.int32, dev)
        _shaped(offsets, "offsets", (B + 1,))
    return B, width, table.stride(0)


def _kv(cache, k, v, dtype):
    index, shape = cache.index, (k.shape[0], cache.heads, cache.dim)
    for t, name in ((k, "k"), (v, "v")):
        if not (_plain(t, 3, dtype, index) and t.shape == shape):
            _tensor(t, name, 3, dtype, cache.device)
            _shaped(t, name, shape)


def cache_write(cache: Cache, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                offsets: torch.Tensor | None = None) -> None:
    """New tokens' keys and values into their places.

    ``k``, ``v`` ``[N, heads, D]`` (any strides with a contiguous last dimension),
    the rows of all sequences one behind another: sequence b has the rows
    ``offsets[b]`` .. ``offsets[b + 1]`` - 1 (int32 ``[B + 1]``), or without offsets
    N / B of them.  They are its last tokens: with ``lengths`` (int32 ``[B]``) its
    tokens in all, the new ones among them, the t-th of n rows stands at position i
    = lengths[b] - n + t, in slot i % page_size of page ``table[b, i //
    page_size]`` (int32).  A row whose position is negative, or whose page is not
    one of the cache's, is left out, and rows behind the last sequence too.  No
    slot may be written twice in a call.

    A plain cache takes rows of its own type, others fp32, fp16 and bf16, each
    element rounded once.  A block of 32 that holds an infinity or NaN reads back
    as NaN; finite values read back as finite.
    """
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a tensor [N, heads, D]")
    B, width, stride = _batch(cache, table, lengths, offsets, k.shape[0])
    dtype = cache.dtype or k.dtype
    _kv(cache, k, v, dtype)
    rows = _pack(_ROWS, B, k.shape[0], width, _DTYPES[dtype], stride, *k.stride()[:2], *v.stride()[:2])
    _check(_call(load().dconv_cache_write, k, cache._shape, rows, k.data_ptr(), v.data_ptr(),
                 *cache._pointers(), table.data_ptr(), lengths.data_ptr(), _ptr(offsets)))


def cache_read(cache: Cache, rows: int, table: torch.Tensor, lengths: torch.Tensor,
               offsets: torch.Tensor | None = None, *, dtype: torch.dtype | None = None,
               out: tuple[torch.Tensor, torch.Tensor] | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """``(k, v)``, ``[rows, heads, D]``: the last tokens of each sequence back, the
    rows that ``cache_write`` with the same ``table``, ``lengths`` and ``offsets``
    wrote (whole sequences where a sequence has as many rows as tokens), rounded to
    ``dtype`` (a plain cache's own, else bf16 if not given).  Zeros for a row whose
    position is negative or whose page is not one of the cache's.  Rows behind the
    last sequence are left as they were (in ``out``, else of no meaning).
    """
    if rows < 0:
        raise ValueError("rows must be 0 or more, got %d" % rows)
    B, width, stride = _batch(cache, table, lengths, offsets, rows)
    if dtype is None:
        dtype = cache.dtype or (out[0].dtype if out is not None else torch.bfloat16)
    if dtype not in _DTYPES or cache.dtype not in (None, dtype):
        raise ValueError("a cache of %s does not read back as %s"
                         % (cache.dtype or ("e4m3" if cache.format == _E4M3 else "e2m1"), dtype))
    if out is None:
        k, v = (torch.empty((rows, cache.heads, cache.dim), dtype=dtype, device=cache.device) for _ in range(2))
    else:
        k, v = out
        if not isinstance(k, torch.Tensor) or k.dim() != 3 or k.shape[0] != rows:
            raise ValueError("out must be two tensors [rows, heads, D]")
        _kv(cache, k, v, dtype)
    shape = _pack(_ROWS, B, rows, width, _DTYPES[dtype], stride, *k.stride()[:2], *v.stride()[:2])
    _check(_call(load().dconv_cache_read, cache.k, cache._shape, shape, *cache._pointers(), table.data_ptr(),
                 lengths.data_ptr(), _ptr(offsets), k.data_ptr(), v.data_ptr()))
    return k, v


def attend_cache(q: torch.Tensor, cache: Cache, table: torch.Tensor, lengths: torch.Tensor,
                 offsets: torch.Tensor | None = None, *, left: int = -1, right: int = 0, sinks: int = 0,
                 scale: float | None = None, max_rows: int | None = None, out: torch.Tensor | None = None,
                 return_lse: bool = False):
    """``attend`` of new tokens over what a cache holds of their sequences.

    ``q[N, Hq, D]``, Hq a multiple of the cache's heads; ``table``, ``lengths`` and
    ``offsets`` as for ``cache_write``, which comes first: the new tokens see
    themselves.  A query at position i sees key j < lengths[b] if j <= i +
    ``right`` and (j >= i - ``left`` or j < ``sinks``); -1 is no limit.  A key whose
    page is not one of the cache's is not seen; a query that sees none gives 0.
    ``scale`` defaults to 1 / sqrt(D).

    ``max_rows``: no sequence has more rows than this (a longer one is left out);
    by it a call of few rows each is one launch less.  Without offsets it is N / B.

    Returns ``out[N, Hq, D]``; with ``return_lse`` also the logarithms of the softmax
    sums, fp32 ``[N, Hq]``.  Rows behind the last sequence, and those of a sequence
    longer than ``max_rows``, are left as they were in the ``out`` that was passed, and
    are of no meaning in tensors that the call makes.  ``out`` must not overlap ``q``.
    """
    if not isinstance(q, torch.Tensor):
        raise ValueError("q must be a torch.Tensor")
    if q.dim() != 3:
        raise ValueError("q must have 3 dimensions, got %d" % q.dim())
    N, Hq, D = size = q.shape
    B, width, stride = _batch(cache, table, lengths, offsets, N)
    dtype = cache.dtype or q.dtype
    if not _plain(q, 3, dtype, cache.index) or dtype not in _DTYPES:
        _tensor(q, "q", 3, None, cache.device)
        _tensor(q, "q", 3, dtype, cache.device)
    if D != cache.dim:
        _shaped(q, "q", (N, Hq, cache.dim))
    if Hq < 1 or Hq % cache.heads:
        raise ValueError("%d query heads do not share %d key heads" % (Hq, cache.heads))
    if left < -1 or right < -1 or sinks < 0:
        raise ValueError("left and right must be -1 (no limit) or more, sinks 0 or more")
    if max_rows is not None and max_rows < 1:
        raise ValueError("max_rows must be 1 or more")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif not (_plain(out, 3, dtype, cache.index) and out.shape == size):
        _tensor(out, "out", 3, dtype, cache.device)
        _shaped(out, "out", size)
    most = max_rows or 0
    if offsets is None and B:
        most = N // B
    shape = _pack(_ATTEND, B, N, width, Hq, _DTYPES[dtype], left, right, sinks, min(most, N),
                  1.0 / math.sqrt(D) if scale is None else scale, stride, *q.stride()[:2], *out.stride()[:2])
    lse = torch.empty((N, Hq), dtype=torch.float32, device=q.device) if return_lse else None
    lib = load()
    ws, n = _workspace(lambda s, size: lib.dconv_cache_attend_workspace(cache._shape, s, size), shape, q.device)
    _check(_call(lib.dconv_cache_attend, q, cache._shape, shape, q.data_ptr(), *cache._pointers(),
                 table.data_ptr(), lengths.data_ptr(), _ptr(offsets), out.data_ptr(), _ptr(lse), _ptr(ws), n))
    return (out, lse) if return_lse else out
