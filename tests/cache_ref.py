"""Plain forms (torch on the CPU) of a cache in pages: what its bits stand for,
which bits a value has, and where a token is."""
import torch

import token_ref as ref

SCALE = torch.float8_e8m0fnu
LARGEST = {"e4m3": 448.0, "e2m1": 6.0}
GRID = {
    "e4m3": torch.tensor([m / 8 * 2.0 ** -6 for m in range(8)] +
                         [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1],
                         dtype=torch.float64),
    "e2m1": torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64),
}


def limit(kind, dt):
    """The largest value of the format's mantissa in the rows' type."""
    return (1.875 if kind == "e4m3" else 1.5) * (2.0 ** 15 if dt == torch.float16 else 2.0 ** 127)


def encode(x, kind):
    """Codes (one byte per element, the sign's bit on top: 128 for e4m3, 8 for
    e2m1) and scales' exponents of x [..., D]."""
    dt = x.dtype
    x = x.cpu().double().unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(x).all(-1)
    x = torch.nan_to_num(x, 0.0, 0.0, 0.0).clamp(-limit(kind, dt), limit(kind, dt))
    top = x.abs().amax(-1)
    s = torch.full_like(top, -127.0)
    for e in range(-127, 128):
        s = torch.where(LARGEST[kind] * 2.0 ** (e - 1) < top, float(e), s)
    s = s.clamp(min=-127.0)
    y = x / torch.exp2(s)[..., None]
    grid = GRID[kind]
    a = y.abs().contiguous()
    hi = torch.searchsorted(grid, a).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    place = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = place + torch.signbit(y).long() * (128 if kind == "e4m3" else 8)
    return code.flatten(-2).to(torch.uint8), torch.where(bad, 255.0, s + 127).to(torch.uint8), bad


def stored(code, kind):
    """Codes as a cache's elements."""
    if kind == "e4m3":
        return code.view(torch.float8_e4m3fn)
    return code[..., 0::2] | code[..., 1::2] << 4


def decode(x, scale, kind):
    """Elements of a cache as 64-bit values."""
    if kind not in LARGEST:
        return x.cpu().double()
    bits = x.cpu().view(torch.uint8)
    if kind == "e2m1":
        bits = torch.stack([bits & 15, bits >> 4], -1).flatten(-2)
    half = 128 if kind == "e4m3" else 8
    place = (bits % half).long()
    grid = torch.cat([GRID[kind], torch.full((half - len(GRID[kind]),), float("nan"), dtype=torch.float64)])
    value = grid[place] * (1.0 - 2.0 * (bits >= half).double())
    e = scale.cpu().view(torch.uint8).double()
    s = torch.where(e == 255, float("nan"), torch.exp2(e - 127))
    return value * s.repeat_interleave(32, -1)


def places(table, lengths, rows, page, pages):
    """For each row its (page, slot), None where it has none."""
    at = []
    for b, (n, r) in enumerate(zip(lengths, rows)):
        n = min(max(n, 0), table.shape[1] * page)
        for i in range(n - r, n):
            p = int(table[b, i // page]) if i >= 0 else -1
            at.append((p, i % page) if i >= 0 and 0 <= p < pages else None)
    return at


class Attend:
    """attend_cache in 64 bits, sequence by sequence, with the bounds of ``attend``:
    out, out_tol, lse, lse_tol, empty for the rows of the sequences."""

    def __init__(self, q, k, v, k_scale, v_scale, kind, table, lengths, rows, left=-1, right=0, sinks=0,
                 scale=None):
        page, pages = k.shape[1], k.shape[0]
        K, V = decode(k, k_scale, kind), decode(v, v_scale, kind)
        table = table.cpu()
        parts, at = [], 0
        for b, (n, r) in enumerate(zip(lengths, rows)):
            n = min(max(n, 0), table.shape[1] * page)
            j = torch.arange(n)
            where = table[b, j // page].long()
            there = (where >= 0) & (where < pages)
            kb, vb = (x[where.clamp(0, pages - 1), j % page] for x in (K, V))
            # keys without a page are taken out; positions stay
            keep = there.nonzero().flatten()
            parts.append(self._sequence(q[at:at + r], kb, vb, keep, n, left, right, sinks, scale))
            at += r
        for i, name in enumerate(("out", "out_tol", "lse", "lse_tol", "empty")):
            setattr(self, name, torch.cat([p[i] for p in parts]))

    @staticmethod
    def _sequence(q, k, v, keep, n, left, right, sinks, scale):
        r, Hq, D = q.shape
        empty = torch.ones((r, Hq), dtype=torch.bool)
        zero = torch.zeros((r, Hq), dtype=torch.float64)
        if r == 0 or n == 0:
            return torch.zeros((r, Hq, D), dtype=torch.float64), ref.TINY[q.dtype] * torch.ones(r, Hq, D).double(), zero, zero, empty
        visible = ref.visible

        def only(*args):
            see = visible(*args)
            gone = torch.ones(n, dtype=torch.bool)
            gone[keep] = False
            see[..., gone] = False
            return see
        ref.visible = only
        try:
            a = ref.Attend(q[None], k[None], v[None], left=left, right=right, sinks=sinks, scale=scale)
        finally:
            ref.visible = visible
        turn = (lambda x: x[0].transpose(0, 1))
        tol = a.out_tol[0]
        if q.dtype == torch.float16:
            # Probabilities below fp16's normal values, as operands, are off by up to half
            # its smallest step, 2^-25, whatever their size.  They are taken against a base
            # that is at most the row's largest score, so their sum l is 1 or more, and the
            # result is off by 2^-25 / l per seen key's value at most.
            seen = torch.einsum("rn,nhd->rhd", a.see[0].double(), v.abs().nan_to_num(0.0))
            tol = tol + 2.0 ** -25 * seen.repeat_interleave(Hq // v.shape[1], 1)
        return (a.out[0], tol, torch.where(turn(a.empty), 0.0, turn(a.lse)),
                torch.where(turn(a.empty), 0.0, turn(a.lse_tol)), turn(a.empty))
