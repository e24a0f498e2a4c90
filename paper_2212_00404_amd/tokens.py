"""Binding of the operators of an attention block over a map's tokens:
``attend`` (windowed attention with first keys that stay visible), ``rotate``
(rotary positions with several axes) and ``join`` (the norms before and after a
block with its gate, scales and residual sum), and their gradients.

Argument marshalling only, as in ``dconv.py``: every computation runs in the
HIP kernels of ``libdconv.so`` (``include/dconv.h`` has the definitions); this
module checks the tensors, allocates outputs and workspaces on the current
torch stream and passes device pointers.  fp32, fp16 and bf16.

Nothing here is recorded by autograd: results do not require gradients, whatever
the arguments do.  The gradients are calls of their own, which the caller makes or
wraps in a ``torch.autograd.Function`` (``examples/token_block.py`` has one for each).
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from .dconv import _call, _check, load

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_NORMS = {"rms": 0, "layer": 1}
_POST_WEIGHT, _GATE, _PRE_WEIGHT, _PRE_BIAS = 1, 2, 4, 8

# The C structs of include/dconv.h, packed (a ctypes.Structure with its arrays
# takes several times as long to fill, which a small call would feel).
_ROTATE_SHAPE = struct.Struct("@9i9q")
_JOIN_SHAPE = struct.Struct("@8i3f8q")
_ATTEND_SHAPE = struct.Struct("@10if15q")


def _pack(layout: struct.Struct, *values) -> bytes:
    try:
        return layout.pack(*values)
    except struct.error as e:
        raise ValueError("a size or an option is not a whole number of 32 bits (%s)" % e) from None


def _tensor(t, name: str, ndim: int, dtype=None, device=None):
    """A tensor of ``ndim`` dimensions on a HIP device whose last dimension is
    contiguous."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch.Tensor" % name)
    if dtype is None:
        if t.dtype not in _DTYPES:
            raise ValueError("%s must be float32, float16 or bfloat16, got %s" % (name, t.dtype))
    elif t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be on a HIP device, got %s" % (name, t.device))
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s, got %s" % (name, device, t.device))
    if t.dim() != ndim:
        raise ValueError("%s must have %d dimensions, got %d" % (name, ndim, t.dim()))
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)


def _plain(t, ndim: int, dtype, index: int) -> bool:
    """What ``_tensor`` asks for, without its messages (a small call is bound by
    the host)."""
    return (isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_cuda and t.get_device() == index
            and t.dim() == ndim and (t.stride(-1) == 1 or t.shape[-1] <= 1))


def _shaped(t, name: str, shape):
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %r, got %r" % (name, tuple(shape), tuple(t.shape)))


def _workspace(query, shape: bytes, device):
    n = ctypes.c_longlong(0)
    _check(query(shape, ctypes.byref(n)))
    n = n.value
    if n == 0:
        return None, 0
    return torch.empty(n, dtype=torch.uint8, device=device), n


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------------------
# rotate
# ---------------------------------------------------------------------------
def rotate(x: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, axis: torch.Tensor, *,
           adjacent: bool = False, inverse: bool = False,
           out: torch.Tensor | None = None) -> torch.Tensor:
    """Rotary positions with several axes.

    ``x[B, T, H, D]`` (any strides with a contiguous last dimension: the query
    and key heads of a fused projection are one call); ``positions[axes, B, T]``
    or ``[axes, T]``, fp32; ``freq[R]`` fp32 and ``axis[R]`` int32, 2 R <= D: the
    frequency and the axis of each pair (``rotary_table`` makes both).  Pair r is
    elements (2r, 2r+1) if ``adjacent``, else (r, r+R); the rest of a head is
    copied.  ``inverse`` turns back, which is the gradient: ``dx = rotate(dy, ...,
    inverse=True)``.  ``out`` may be ``x``.
    """
    _tensor(x, "x", 4)
    dev, index = x.device, x.get_device()
    B, T, H, D = x.shape
    if isinstance(positions, torch.Tensor) and positions.dim() == 2:
        positions = positions[:, None].expand(-1, B, -1)
    if not (isinstance(positions, torch.Tensor) and positions.dtype is torch.float32
            and positions.get_device() == index and positions.dim() == 3):
        raise ValueError("positions must be a float32 tensor [axes, B, T] or [axes, T] on %s" % dev)
    axes, Bp, Tp = positions.shape
    if axes < 1:
        raise ValueError("positions must have an axis")
    if Bp != B or Tp != T:
        _shaped(positions, "positions", (axes, B, T))
    if not (_plain(freq, 1, torch.float32, index) and _plain(axis, 1, torch.int32, index)):
        _tensor(freq, "freq", 1, torch.float32, dev)
        _tensor(axis, "axis", 1, torch.int32, dev)
    R = freq.shape[0]
    if axis.shape[0] != R:
        _shaped(axis, "axis", (R,))
    if 2 * R > D:
        raise ValueError("%d pairs do not fit a head of %d" % (R, D))
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif out is not x:
        _tensor(out, "out", 4, x.dtype, dev)
        _shaped(out, "out", x.shape)
    shape = _pack(_ROTATE_SHAPE, B, T, H, D, R, axes, bool(adjacent), bool(inverse), _DTYPES[x.dtype],
                  *x.stride()[:3], *out.stride()[:3], *positions.stride())
    _check(_call(load().dconv_rotate, x, shape, x.data_ptr(), positions.data_ptr(), freq.data_ptr(),
                 axis.data_ptr(), out.data_ptr()))
    return out


def rotary_table(pairs, base: float = 10000.0, interleaved: bool = False, device=None):
    """``(freq, axis)`` for ``rotate``: ``pairs[a]`` pairs turn by axis ``a``, the
    i-th of them by ``base ** (-i / pairs[a])`` radians per unit of position.
    The axes' pairs stand one block after another, or dealt out in turn
    (``interleaved``)."""
    entries = [[(base ** (-i / n), a) for i in range(n)] for a, n in enumerate(pairs)]
    if interleaved:
        order = [e[i] for i in range(max(map(len, entries), default=0)) for e in entries if i < len(e)]
    else:
        order = [p for e in entries for p in e]
    return (torch.tensor([f for f, _ in order], dtype=torch.float32, device=device),
            torch.tensor([a for _, a in order], dtype=torch.int32, device=device))


def map_positions(frames: int, rows: int, cols: int, device=None) -> torch.Tensor:
    """``[3, frames * rows * cols]``: time, row and column of each token of a clip
    of maps read row by row."""
    grid = torch.meshgrid(torch.arange(frames), torch.arange(rows), torch.arange(cols), indexing="ij")
    return torch.stack(grid).reshape(3, -1).to(device=device, dtype=torch.float32)


# ---------------------------------------------------------------------------
# join
# ---------------------------------------------------------------------------
def _join_arguments(branch, x, norm, post, post_weight, gate, pre_weight, pre_bias, residual_scale,
                    branch_scale, eps, dh=None, dy=None):
    """Checks, and the C struct."""
    _tensor(x, "x", 3)
    dtype, index, size = x.dtype, x.get_device(), x.shape
    B, T, D = size
    if norm not in _NORMS:
        raise ValueError("norm must be one of %s" % sorted(_NORMS))
    strides = []
    for t, name in ((branch, "branch"), (x, "x"), (dh, "dh"), (dy, "dy")):
        if t is None:
            strides += (0, 0)
            continue
        if t is not x and not (_plain(t, 3, dtype, index) and t.shape == size):
            _tensor(t, name, 3, dtype, x.device)
            _shaped(t, name, size)
        strides += t.stride()[:2]
    if branch is None and (gate is not None or post_weight is not None):
        raise ValueError("gate and post_weight need a branch")
    if post_weight is not None and not post:
        raise ValueError("post_weight needs post=True")
    per, vt = 0, None
    for t, name, bit in ((post_weight, "post_weight", _POST_WEIGHT), (gate, "gate", _GATE),
                         (pre_weight, "pre_weight", _PRE_WEIGHT), (pre_bias, "pre_bias", _PRE_BIAS)):
        if t is None:
            continue
        if not (isinstance(t, torch.Tensor) and (t.dtype is torch.float32 or t.dtype is dtype)
                and t.is_cuda and t.get_device() == index and t.is_contiguous()):
            raise ValueError("%s must be a contiguous tensor of float32 or %s on %s" % (name, dtype, x.device))
        if vt is None:
            vt = t.dtype
        elif t.dtype is not vt:
            raise ValueError("the vectors must have one type")
        shape = t.shape
        if len(shape) == 2 and shape[0] == B and shape[1] == D:
            per |= bit
        elif len(shape) != 1 or shape[0] != D:
            raise ValueError("%s must be %r or %r, got %r" % (name, (D,), (B, D), tuple(shape)))
    return _pack(_JOIN_SHAPE, B, T, D, _DTYPES[dtype], _DTYPES[vt or dtype], _NORMS[norm],
                 bool(post and branch is not None), per, residual_scale, branch_scale, eps, *strides)


def join(branch: torch.Tensor | None, x: torch.Tensor, *, norm: str = "rms", post: bool = False,
         post_weight=None, gate=None, pre_weight=None, pre_bias=None, residual_scale: float = 1.0,
         branch_scale: float = 1.0, eps: float = 1e-6, pre: bool = True, return_stats: bool = False):
    """From a block's output to the next block's input::

        p = N(branch) * post_weight  if post else  branch
        h = residual_scale * x + branch_scale * gate * p
        y = N(h) * pre_weight + pre_bias

    N is the norm of the last dimension, ``"rms"`` or ``"layer"``.  ``branch`` and
    ``x`` are ``[B, T, D]``; each vector is ``[D]`` or, set for each sequence,
    ``[B, D]``, of ``x``'s type or fp32, or None (left out).

    Returns ``(h, y)``, y None with ``pre=False`` (after the last block), h None
    without a ``branch`` (the norm before the first block, of residual_scale * x);
    with ``return_stats`` also the rows' statistics, which ``join_backward`` takes.
    """
    shape = _join_arguments(branch, x, norm, post, post_weight, gate, pre_weight, pre_bias,
                            residual_scale, branch_scale, eps)
    if branch is None and not pre:
        raise ValueError("nothing to compute: no branch and pre=False")
    if not pre and (pre_weight is not None or pre_bias is not None):
        raise ValueError("pre_weight and pre_bias need pre=True")
    h = None if branch is None else torch.empty_like(x, memory_format=torch.contiguous_format)
    y = torch.empty_like(x, memory_format=torch.contiguous_format) if pre else None
    stats = torch.empty((*x.shape[:2], 4), dtype=torch.float32, device=x.device) if return_stats else None
    _check(_call(load().dconv_join, x, shape, _ptr(branch), x.data_ptr(), _ptr(post_weight), _ptr(gate),
                 _ptr(pre_weight), _ptr(pre_bias), _ptr(h), _ptr(y), _ptr(stats)))
    return (h, y, stats) if return_stats else (h, y)


def join_backward(dh, dy, branch, x: torch.Tensor, stats: torch.Tensor, *, norm: str = "rms",
                  post: bool = False, post_weight=None, gate=None, pre_weight=None, pre_bias=None,
                  residual_scale: float = 1.0, branch_scale: float = 1.0, eps: float = 1e-6) -> dict:
    """Gradients of ``join`` for those of its outputs, ``dh`` and ``dy`` (None:
    zeros).  The other arguments are the forward call's.  Returns a dict with
    ``"x"`` and an entry for ``branch`` and each vector that was given, in its
    shape and type."""
    shape = _join_arguments(branch, x, norm, post, post_weight, gate, pre_weight, pre_bias,
                            residual_scale, branch_scale, eps, dh, dy)
    _tensor(stats, "stats", 3, torch.float32, x.device)
    _shaped(stats, "stats", (x.shape[0], x.shape[1], 4))
    if not stats.is_contiguous():
        raise ValueError("stats must be contiguous")
    grads = {}
    if branch is not None:
        grads["branch"] = torch.empty_like(x, memory_format=torch.contiguous_format)
    grads["x"] = torch.empty_like(x, memory_format=torch.contiguous_format)
    for t, name in ((post_weight, "post_weight"), (gate, "gate"), (pre_weight, "pre_weight"),
                    (pre_bias, "pre_bias")):
        if t is not None:
            grads[name] = torch.empty_like(t)
    lib = load()
    ws, n = _workspace(lib.dconv_join_workspace, shape, x.device)
    _check(_call(lib.dconv_join_backward, x, shape, _ptr(dh), _ptr(dy), _ptr(branch), x.data_ptr(),
                 _ptr(post_weight), _ptr(gate), _ptr(pre_weight), stats.data_ptr(),
                 _ptr(grads.get("branch")), grads["x"].data_ptr(), _ptr(grads.get("post_weight")),
                 _ptr(grads.get("gate")), _ptr(grads.get("pre_weight")), _ptr(grads.get("pre_bias")),
                 _ptr(ws), n))
    return grads


# ---------------------------------------------------------------------------
# attend
# ---------------------------------------------------------------------------
def _attend_arguments(q, k, v, left, right, sinks, scale, lengths, starts, out, dout=None):
    _tensor(q, "q", 4)
    dt, dev, index = q.dtype, q.device, q.get_device()
    B, Tq, Hq, D = size = q.shape
    if not (_plain(k, 4, dt, index) and _plain(v, 4, dt, index)):
        _tensor(k, "k", 4, dt, dev)
        _tensor(v, "v", 4, dt, dev)
    Bk, Tk, Hkv, Dk = k.shape
    if Bk != B or Dk != D or v.shape != k.shape:
        _shaped(k, "k", (B, Tk, Hkv, D))
        _shaped(v, "v", k.shape)
    if Hkv < 1 or Hq % Hkv:
        raise ValueError("%d query heads do not share %d key heads" % (Hq, Hkv))
    if left < -1 or right < -1 or sinks < 0:
        raise ValueError("left and right must be -1 (no limit) or more, sinks 0 or more")
    for t, name in ((lengths, "lengths"), (starts, "starts")):
        if t is not None and not (_plain(t, 1, torch.int32, index) and t.shape[0] == B):
            _tensor(t, name, 1, torch.int32, dev)
            _shaped(t, name, (B,))
    for t, name in ((out, "out"), (dout, "dout")):
        if t is not None and not (_plain(t, 4, dt, index) and t.shape == size):
            _tensor(t, name, 4, dt, dev)
            _shaped(t, name, size)
    return _pack(
        _ATTEND_SHAPE, B, Tq, Tk, Hq, Hkv, D, _DTYPES[dt], left, right, sinks,
        1.0 / math.sqrt(D) if scale is None else scale, *q.stride()[:3], *k.stride()[:3],
        *v.stride()[:3], *out.stride()[:3], *((0, 0, 0) if dout is None else dout.stride()[:3]))


def attend(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, left: int = -1, right: int = 0,
           sinks: int = 0, scale: float | None = None, lengths: torch.Tensor | None = None,
           starts: torch.Tensor | None = None, out: torch.Tensor | None = None,
           return_lse: bool = False):
    """Softmax attention in which a query sees a window and the first keys.

    ``q[B, Tq, Hq, D]``, ``k``, ``v`` ``[B, Tk, Hkv, D]`` (any strides with a
    contiguous last dimension; Hq a multiple of Hkv).  The query t of sequence b
    stands at position i = ``starts[b]`` + t and sees key j < ``lengths[b]`` if
    j <= i + ``right`` and (j >= i - ``left`` or j < ``sinks``); -1 is no limit, a
    negative position sees nothing.  ``lengths`` (int32 ``[B]``) defaults to Tk,
    ``starts`` to lengths - Tq: the queries are the last tokens, as new tokens
    over a cache are.  For whole sequences padded to one length pass starts of 0.
    ``scale`` defaults to 1 / sqrt(D).  A query that sees no key gives 0.

    Returns ``out[B, Tq, Hq, D]``; with ``return_lse`` also the logarithms of the
    softmax sums, fp32 ``[B, Hq, Tq]``, which ``attend_backward`` takes.
    """
    if out is None:
        if not isinstance(q, torch.Tensor):
            raise ValueError("q must be a torch.Tensor")
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    shape = _attend_arguments(q, k, v, left, right, sinks, scale, lengths, starts, out)
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device) \
        if return_lse else None
    lib = load()
    ws, n = _workspace(lib.dconv_attend_workspace, shape, q.device)
    _check(_call(lib.dconv_attend, q, shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths),
                 _ptr(starts), out.data_ptr(), _ptr(lse), _ptr(ws), n))
    return (out, lse) if return_lse else out


def attend_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                    out: torch.Tensor, lse: torch.Tensor, *, left: int = -1, right: int = 0,
                    sinks: int = 0, scale: float | None = None, lengths: torch.Tensor | None = None,
                    starts: torch.Tensor | None = None):
    """``(dq, dk, dv)`` of ``attend`` for the gradient ``dout`` of its output.
    ``out`` and ``lse`` are what it returned, the other arguments what it took.
    (Heads of more than 128 are some hundred times slower.)"""
    _tensor(dout, "dout", 4)
    shape = _attend_arguments(q, k, v, left, right, sinks, scale, lengths, starts, out, dout)
    _tensor(lse, "lse", 3, torch.float32, q.device)
    _shaped(lse, "lse", (q.shape[0], q.shape[2], q.shape[1]))
    if not lse.is_contiguous():
        raise ValueError("lse must be contiguous")
    dq, dk, dv = (torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v))
    lib = load()
    ws, n = _workspace(lib.dconv_attend_backward_workspace, shape, q.device)
    _check(_call(lib.dconv_attend_backward, q, shape, dout.data_ptr(), q.data_ptr(), k.data_ptr(),
                 v.data_ptr(), out.data_ptr(), lse.data_ptr(), _ptr(lengths), _ptr(starts),
                 dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), n))
    return dq, dk, dv
