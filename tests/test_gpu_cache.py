"""GPU: a cache in pages, what is written to it, read from it and attended over,
against the definitions in 64 bits."""
import math
import os
import sys

import pytest
import torch

import cache_ref as cref
import paper_2212_00404_amd as dc
import token_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
TYPE_IDS = ["f32", "f16", "bf16"]
KINDS = ["plain", "e4m3", "e2m1"]


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


class Pool:
    """A cache of random contents, a table, and the sizes of its sequences."""

    def __init__(self, seed, dt, kind, rows, lengths, Hkv, D, page, spare=2, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.dt, self.rows, self.lengths, self.page, self.D, self.Hkv = kind, dt, rows, lengths, page, D, Hkv
        held = [-(-n // page) for n in lengths]
        self.pages = sum(held) + spare
        order = torch.randperm(self.pages, generator=g).int()
        self.table = torch.full((len(rows), max(held + [1])), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        parts = []
        for _ in range(2):
            x = (torch.randn(self.pages, Hkv, page, D, generator=g) * spread).to(dt)
            if kind == "plain":
                parts.append((x, None))
            else:
                code, scale, _ = cref.encode(x, kind)
                parts.append((cref.stored(code, kind), scale.view(cref.SCALE)))
        (self.k, self.ks), (self.v, self.vs) = (
            tuple(None if t is None else t.to(DEV).transpose(1, 2) for t in p) for p in parts)
        self.cache = dc.Cache(self.k, self.v, self.ks, self.vs)
        self.where = (self.table.to(DEV), ints(lengths), ints([sum(rows[:b]) for b in range(len(rows) + 1)]))

    def queries(self, seed, Hq, tail=0):
        g = torch.Generator().manual_seed(seed)
        return torch.randn(sum(self.rows) + tail, Hq, self.D, generator=g).to(self.dt).to(DEV)

    def reference(self, q, **how):
        return cref.Attend(q.cpu(), self.k.cpu(), self.v.cpu(), None if self.ks is None else self.ks.cpu(),
                           None if self.vs is None else self.vs.cpu(), self.kind, self.table, self.lengths, self.rows,
                           **how)


def check(out, lse, want):
    n = want.out.shape[0]
    ref.check(out[:n], want.out, want.out_tol, "out")
    if lse is not None:
        lse = lse[:n].cpu().double()
        assert (lse[want.empty] == -math.inf).all()
        ref.check(torch.where(want.empty, 0.0, lse), torch.where(want.empty, 0.0, want.lse), want.lse_tol, "lse")


def compare(pool, Hq, seed=50, **how):
    q = pool.queries(seed, Hq)
    out, lse = dc.attend_cache(q, pool.cache, *pool.where, return_lse=True, **how)
    torch.cuda.synchronize()
    check(out, lse, pool.reference(q, **how))
    return out


# ---------------------------------------------------------------------------
# writing and reading back
# ---------------------------------------------------------------------------
# rows, lengths, heads, head size, page size
MOVED = [
    ([1], [1], 1, 32, 1),
    ([1, 1, 1], [5, 64, 17], 2, 64, 16),
    ([7, 0, 1, 40], [7, 3, 90, 41], 3, 96, 24),
    ([130, 5], [131, 700], 8, 128, 64),
    ([33, 2, 0], [64, 2, 0], 1, 256, 5),
]
PLAIN_MOVED = [([3, 9], [4, 30], 2, 1, 4), ([20, 1, 6], [33, 1, 50], 3, 81, 7), ([66], [66], 6, 80, 24)]


def contents(kind, shape, dt, g):
    """Values of very different sizes, blocks of zeros, of the smallest and of the
    largest values, and values half-way between two codes."""
    x = torch.randn(shape, generator=g, dtype=torch.float64)
    x = x * torch.exp2(torch.randint(-12, 12, (*shape[:-1], 1), generator=g).double())
    flat = x.view(-1, shape[-1])
    for i in range(0, flat.shape[0], 5):
        what = (i // 5) % 5
        if what == 0:
            flat[i] = 0.0
        elif what == 1:
            flat[i] = torch.sign(flat[i]) * torch.finfo(dt).max * (1 - torch.rand(shape[-1], generator=g).double() / 3)
        elif what == 2:
            flat[i] = torch.sign(flat[i]) * torch.finfo(dt).tiny * torch.rand(shape[-1], generator=g).double() * 3
        elif kind != "plain":
            grid = cref.GRID[kind]
            at = torch.randint(0, len(grid) - 1, (shape[-1],), generator=g)
            flat[i] = (grid[at] + grid[at + 1]) / 2 * torch.sign(flat[i]) * 2.0 ** (what - 6)
            flat[i, 0] = cref.LARGEST[kind] * 2.0 ** (what - 6) * (1 + (what == 4) * 2.0 ** -7)
    return x.to(dt)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("kind, case", [(n, c) for n in KINDS for c in MOVED + (PLAIN_MOVED if n == "plain" else [])],
                         ids=str)
def test_write_and_read(kind, case, dt):
    rows, lengths, H, D, page = case
    pool = Pool(1, dt, kind, rows, lengths, H, D, page)
    N, tail = sum(rows), 3
    g = torch.Generator().manual_seed(2)
    k, v = (contents(kind, (N + tail, H, D), dt, g) for _ in range(2))
    before = [None if t is None else t.clone() for t in (pool.k, pool.v, pool.ks, pool.vs)]
    dc.cache_write(pool.cache, k.to(DEV), v.to(DEV), *pool.where)
    torch.cuda.synchronize()
    at = cref.places(pool.table, lengths, rows, page, pool.pages)
    assert None not in at
    for x, kept, scale, b0, s0 in ((k, pool.k, pool.ks, before[0], before[2]), (v, pool.v, pool.vs, before[1], before[3])):
        if kind == "plain":
            want, ws = x, None
        else:
            code, ws, _ = cref.encode(x, kind)
            want = cref.stored(code, kind)
        full = b0.cpu().clone()
        raw = (lambda t: t.contiguous().view(torch.uint8))
        for r, (p, s) in enumerate(at):
            full[p, s] = want[r]
        assert torch.equal(raw(kept.cpu()), raw(full))
        if ws is not None:
            fs = s0.cpu().contiguous().view(torch.uint8).clone()
            for r, (p, s) in enumerate(at):
                fs[p, s] = ws[r]
            assert torch.equal(raw(scale.cpu()), fs)
    # back: what the bits stand for, rounded once; rows behind the last as they were
    for to in ([dt] if kind == "plain" else TYPES):
        out = tuple(torch.full((N + tail, H, D), 7.0, dtype=to, device=DEV) for _ in range(2))
        dc.cache_read(pool.cache, N + tail, *pool.where, out=out)
        torch.cuda.synchronize()
        for o, kept, scale in zip(out, (pool.k, pool.v), (pool.ks, pool.vs)):
            dense = cref.decode(kept, scale, kind).to(to)
            want = torch.stack([dense[p, s] for p, s in at]) if at else torch.empty((0, H, D), dtype=to)
            assert torch.equal(o[:N].cpu(), want)
            assert (o[N:] == 7.0).all()


@pytest.mark.parametrize("kind", KINDS)
def test_moves_of_more_sequences_than_lds_holds(kind):
    """Offsets and lengths looked up in memory: 700 sequences, some without rows."""
    dt = torch.bfloat16
    rows = [(b * 5) % 4 for b in range(700)]
    lengths = [r + (b * 31) % 40 for b, r in enumerate(rows)]
    pool = Pool(17, dt, kind, rows, lengths, 1, 32, 8)
    N = sum(rows)
    g = torch.Generator().manual_seed(18)
    k, v = (torch.randn(N, 1, 32, generator=g).to(dt) for _ in range(2))
    dc.cache_write(pool.cache, k.to(DEV), v.to(DEV), *pool.where)
    got = dc.cache_read(pool.cache, N, *pool.where, dtype=dt)
    at = cref.places(pool.table, lengths, rows, 8, pool.pages)
    for x, o, kept, scale in zip((k, v), got, (pool.k, pool.v), (pool.ks, pool.vs)):
        want = x.double()
        if kind != "plain":
            code, s, _ = cref.encode(x, kind)
            want = cref.decode(cref.stored(code, kind), s.view(cref.SCALE), kind)
        assert torch.equal(o.cpu().double(), want)
        dense = cref.decode(kept, scale, kind)
        assert torch.equal(torch.stack([dense[p, i] for p, i in at]), want)
    compare(pool, 2)


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_finite_values_read_back_finite(kind):
    """Up to the type's largest; each within half a step of its block's scale."""
    for dt in TYPES:
        pool = Pool(3, dt, kind, [4], [4], 1, 64, 4)
        x = torch.full((4, 1, 64), torch.finfo(dt).max, dtype=dt)
        x[1] /= 3
        x[2, 0, ::3] = -torch.finfo(dt).max
        x[3] = torch.finfo(dt).tiny
        dc.cache_write(pool.cache, x.to(DEV), x.to(DEV), *pool.where)
        k, v = dc.cache_read(pool.cache, 4, *pool.where, dtype=dt)
        assert torch.isfinite(k).all() and torch.equal(k, v)
        # a format of m bits of mantissa: 2^-(m+1) relative, and what limiting takes
        # off: up to 1 - L / max < 1 / 16 (1 / 4 in 4 bits)
        off = {"e4m3": 2.0 ** -4, "e2m1": 2.0 ** -2}[kind]
        assert ((k.cpu().double() - x.double()).abs() <= off * x.double().abs()).all()


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_blocks_with_an_infinity_or_nan_read_back_as_nan(kind, dt):
    pool = Pool(4, dt, kind, [3], [9], 2, 96, 8)
    g = torch.Generator().manual_seed(5)
    x = torch.randn(3, 2, 96, generator=g).to(dt)
    x[0, 0, 5], x[1, 1, 64], x[2, 0, 95] = math.inf, math.nan, -math.inf
    dc.cache_write(pool.cache, x.to(DEV), x.to(DEV), *pool.where)
    k, _ = dc.cache_read(pool.cache, 3, *pool.where, dtype=dt)
    bad = torch.zeros(3, 2, 96, dtype=torch.bool)
    bad[0, 0, :32] = bad[1, 1, 64:] = bad[2, 0, 64:] = True
    assert torch.equal(k.isnan().cpu(), bad)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_a_place(kind):
    """Positions before the first token, pages that are none, lengths past the
    table: nothing is written for them, zeros are read; nothing else changes."""
    dt = torch.bfloat16
    rows, lengths = [5, 6, 3, 4], [3, 20, 1000, -4]
    pool = Pool(6, dt, kind, rows, [3, 20, 24, 0], 2, 64, 8)
    pool.table[1, 2], pool.table[2, 2] = pool.pages, -1
    table = pool.table.to(DEV)
    where = (table, ints(lengths), pool.where[2])
    g = torch.Generator().manual_seed(7)
    k = torch.randn(18, 2, 64, generator=g).to(dt).to(DEV)
    before = pool.k.clone()
    dc.cache_write(pool.cache, k, k, *where)
    back, _ = dc.cache_read(pool.cache, 18, *where, dtype=dt)
    at = cref.places(pool.table, lengths, rows, 8, pool.pages)
    assert [a is None for a in at] == [True] * 2 + [False] * 3 + [False] * 2 + [True] * 4 + [True] * 3 + [True] * 4
    dense = cref.decode(pool.k, pool.ks, kind)
    for r, a in enumerate(at):
        want = torch.zeros(2, 64) if a is None else dense[a].to(dt)
        assert torch.equal(back[r].cpu().double(), want.double())
    same = torch.ones(pool.pages, 8, dtype=torch.bool)
    for a in at:
        if a is not None:
            same[a] = False
    raw = (lambda t: t.cpu().contiguous().view(torch.uint8))
    assert torch.equal(raw(pool.k)[same], raw(before)[same])


@pytest.mark.parametrize("kind", KINDS)
def test_strides_and_alignment_of_moves(kind):
    """Rows of a fused projection, heads and slots in another order, pools that
    begin between two words."""
    dt = torch.float16
    rows, lengths, H, D, page = [9, 1, 30], [12, 5, 64], 3, 64, 8
    pool = Pool(8, dt, kind, rows, lengths, H, D, page)
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn(sum(rows), 3 * H, D + 1, generator=g).to(dt).to(DEV)[..., 1:]
    k, v = qkv[:, H:2 * H], qkv[:, 2 * H:]
    dc.cache_write(pool.cache, k, v, *pool.where)

    def other(t):
        if t is None:
            return None
        last = t.shape[-1]
        raw = torch.zeros((page, pool.pages, H, last + 3), dtype=torch.uint8 if t.element_size() == 1 else t.dtype,
                          device=DEV)
        return raw.view(t.dtype).permute(1, 0, 2, 3)[..., 1:1 + last] if t.element_size() == 1 else raw.permute(1, 0, 2, 3)[..., 1:1 + last]
    odd = [other(t) for t in (pool.k, pool.v, pool.ks, pool.vs)]
    cache = dc.Cache(*odd)
    dc.cache_write(cache, k.contiguous(), v, *pool.where)
    at = cref.places(pool.table, lengths, rows, page, pool.pages)
    raw = (lambda t: t.cpu().contiguous().view(torch.uint8))
    for a, b in zip((pool.k, pool.v, pool.ks, pool.vs), odd):
        if a is not None:
            a, b = raw(a), raw(b)
            for p, s in at:
                assert torch.equal(a[p, s], b[p, s])
    want = dc.cache_read(pool.cache, sum(rows), *pool.where, dtype=dt)
    buf = torch.zeros((2, sum(rows), H, D + 1), dtype=dt, device=DEV)[..., 1:]
    got = dc.cache_read(cache, sum(rows), *pool.where, out=(buf[0], buf[1]))
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_as_many_rows_for_each_without_offsets():
    pool = Pool(10, torch.bfloat16, "e4m3", [4, 4, 4], [9, 4, 30], 2, 64, 8)
    table, lengths, offsets = pool.where
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(12, 2, 64, generator=g).bfloat16().to(DEV) for _ in range(2))
    dc.cache_write(pool.cache, k, v, table, lengths, offsets)
    want = dc.cache_read(pool.cache, 12, table, lengths, offsets)
    pool.k.view(torch.uint8).zero_()
    pool.v.view(torch.uint8).zero_()
    dc.cache_write(pool.cache, k, v, table, lengths)
    for a, b in zip(want, dc.cache_read(pool.cache, 12, table, lengths)):
        assert torch.equal(a, b)
    q = pool.queries(12, 4)
    assert torch.equal(dc.attend_cache(q, pool.cache, table, lengths),
                       dc.attend_cache(q, pool.cache, table, lengths, offsets))


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
# rows, lengths, query heads, key heads, head size, page size, window
ATTENDED = [
    ([1], [1], 1, 1, 32, 1, dict()),
    ([1, 1, 1, 1], [1, 700, 33, 128], 8, 2, 64, 16, dict()),
    ([1, 1, 1], [900, 65, 300], 4, 4, 128, 64, dict(left=200, sinks=3)),
    ([5, 2, 0, 1], [400, 2, 9, 1], 7, 1, 96, 24, dict()),
    ([3, 1], [1500, 40], 16, 2, 128, 32, dict(left=600, sinks=40)),
    ([40, 1, 129, 0, 7], [40, 260, 300, 12, 90], 4, 2, 64, 8, dict(left=70, sinks=2)),
    ([200, 33], [500, 33], 6, 2, 128, 128, dict()),
    ([300], [300], 8, 1, 64, 48, dict(left=30, right=30, sinks=1)),
    ([64, 17], [64, 90], 3, 3, 256, 16, dict(right=-1)),
    ([1, 90], [250, 120], 2, 1, 256, 5, dict(left=60)),
    ([150, 150], [150, 400], 2, 2, 32, 200, dict(left=0, right=4)),
]
PLAIN_ATTENDED = [
    ([1, 2, 70], [1, 2, 70], 1, 1, 1, 3, dict()),
    ([9, 1], [77, 130], 6, 3, 40, 16, dict(left=20, sinks=2)),
    ([57, 48, 1], [101, 300, 64], 6, 2, 80, 24, dict(left=50, sinks=1)),
    ([130, 1], [140, 500], 2, 1, 81, 7, dict()),
    ([20, 1], [50, 260], 4, 2, 200, 32, dict()),
]


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("kind, case", [(n, c) for n in KINDS
                                        for c in ATTENDED + (PLAIN_ATTENDED if n == "plain" else [])], ids=str)
def test_attention(kind, case, dt):
    rows, lengths, Hq, Hkv, D, page, how = case
    compare(Pool(20, dt, kind, rows, lengths, Hkv, D, page), Hq, **how)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("rows", [[1, 3], [90, 40]])
def test_scales(rows, scale):
    for kind in KINDS:
        for dt in TYPES:
            compare(Pool(19, dt, kind, rows, [900, 130], 2, 64, 16), 4, scale=scale, left=300)


@pytest.mark.parametrize("kind", KINDS)
def test_many_sequences(kind):
    """More sequences than a wave has lanes, single tokens and chunks, some empty."""
    rows = [(b * 7) % 5 if b % 9 else 40 for b in range(300)]
    lengths = [r + (b * 53) % 290 for b, r in enumerate(rows)]
    compare(Pool(21, torch.bfloat16, kind, rows, lengths, 2, 64, 16), 4)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("rows, length", [(1, 9000), (4, 6001), (40, 5000), (150, 4100)])
def test_long_walks_of_few_rows(rows, length, dt):
    """Keys divided over many workgroups, and joined."""
    kind = {torch.float32: "plain", torch.float16: "e2m1", torch.bfloat16: "e4m3"}[dt]
    compare(Pool(22, dt, kind, [rows, 1], [length, 3], 2, 64, 64), 4)
    compare(Pool(23, dt, kind, [rows], [length], 1, 128, 16), 8, left=length // 2, sinks=7)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_see_nothing(kind):
    """Positions before the first token, sequences without tokens, pages that are
    none, and a window that ends before the first key."""
    dt = torch.bfloat16
    for rows, lengths in (([4, 3, 2, 50], [0, 1, 2, 20]), ([1, 1, 2, 1], [0, 1, 0, 9])):
        pool = Pool(24, dt, kind, rows, lengths, 2, 64, 8)
        out = compare(pool, 4)
        assert (out[:rows[0]] == 0).all()
        pool.table[:, 0] = pool.pages + 5
        pool.where = (pool.table.to(DEV),) + pool.where[1:]
        compare(pool, 4)
        compare(pool, 4, left=3, sinks=2)
        pool.table[:] = -1
        pool.where = (pool.table.to(DEV),) + pool.where[1:]
        assert (compare(pool, 4) == 0).all()


@pytest.mark.parametrize("rows", [[3, 1], [70, 20]])
@pytest.mark.parametrize("kind", KINDS)
def test_pages_that_are_none_inside_a_sequence(kind, rows):
    pool = Pool(25, torch.float16, kind, rows, [333, 90], 2, 64, 16)
    pool.table[0, 3], pool.table[0, 11], pool.table[1, 0] = -1, pool.pages, 1 << 30
    pool.where = (pool.table.to(DEV),) + pool.where[1:]
    compare(pool, 4)
    compare(pool, 4, left=50, sinks=60)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("rows", [[1, 1, 2], [90, 1, 50]])
@pytest.mark.parametrize("kind", KINDS)
def test_what_is_not_seen_does_not_matter(kind, rows, dt):
    """Slots behind a sequence's end, other pages, keys before the window: NaN in
    elements and scales there changes no bit."""
    lengths, page = [301, 18, 77], 16
    pool = Pool(26, dt, kind, rows, lengths, 2, 64, page)
    how = dict(left=40, sinks=3)
    q = pool.queries(27, 4)
    want = dc.attend_cache(q, pool.cache, *pool.where, **how)
    seen = torch.zeros(pool.pages, page, dtype=torch.bool)
    for b, (n, r) in enumerate(zip(lengths, rows)):
        for j in range(n):
            if j < 3 or j >= n - r - 40:
                seen[pool.table[b, j // page], j % page] = True
    hide = ~seen.to(DEV)
    for t in (pool.k, pool.v):
        if kind == "plain":
            t[hide] = math.nan
        else:
            t.view(torch.uint8)[hide] = 0x7F
    for t in (pool.ks, pool.vs):
        if t is not None:
            t.view(torch.uint8)[hide] = 255
    junk = pool.table.clone()
    for b, n in enumerate(lengths):
        junk[b, -(-n // page):] = torch.tensor([-5, 1 << 30, pool.pages])[torch.arange(junk.shape[1] - -(-n // page)) % 3]
    got = dc.attend_cache(q, pool.cache, junk.to(DEV), *pool.where[1:], **how)
    assert torch.equal(want, got)
    check(got, None, pool_reference_without(pool, hide, q, how))


def pool_reference_without(pool, hide, q, how):
    """The reference, with zeros where nothing is seen."""
    k, v = (t.clone() for t in (pool.k, pool.v))
    for t in (k, v):
        (t if pool.kind == "plain" else t.view(torch.uint8))[hide] = 0
    ks, vs = (None if t is None else t.clone() for t in (pool.ks, pool.vs))
    for t in (ks, vs):
        if t is not None:
            t.view(torch.uint8)[hide] = 0
    cpu = (lambda t: None if t is None else t.cpu())
    return cref.Attend(q.cpu(), k.cpu(), v.cpu(), cpu(ks), cpu(vs), pool.kind, pool.table, pool.lengths, pool.rows, **how)


@pytest.mark.parametrize("rows", [[1, 1], [70, 40]])
@pytest.mark.parametrize("kind", KINDS)
def test_nan_reaches_exactly_the_queries_that_see_it(kind, rows):
    dt, lengths, at = torch.bfloat16, [120, 90], 85
    for name in ("k", "v"):
        pool = Pool(28, dt, kind, rows, lengths, 2, 64, 16)
        q = pool.queries(29, 4)
        clean = pool.reference(q, left=30)
        page, slot = int(pool.table[0, at // 16]), at % 16
        if kind == "plain":
            getattr(pool, name)[page, slot, 1, 7] = math.nan
        else:
            getattr(pool, name + "s").view(torch.uint8)[page, slot, 1, 0] = 255
        got = dc.attend_cache(q, pool.cache, *pool.where, left=30)
        bad = torch.zeros(sum(rows), 4, dtype=torch.bool, device=DEV)
        i = torch.arange(lengths[0] - rows[0], lengths[0])
        sees = (i >= at) & (i - 30 <= at)
        bad[:rows[0], 2:] = sees[:, None].to(DEV)
        assert torch.equal(torch.isnan(got).any(-1), bad)
        # (the other rows of a tile are summed by the plain form then: other bits, the
        # same bound)
        ref.check(got[~bad], clean.out[~bad.cpu()], clean.out_tol[~bad.cpu()], "out")


def test_values_whose_sum_passes_the_types_range():
    """Sums before the division pass fp32's range; their mean does not."""
    for rows in ([2], [60]):
        pool = Pool(30, torch.float32, "plain", rows, [700], 1, 64, 16)
        pool.v[:] = 3e38
        q = pool.queries(31, 2) * 0.01
        out = dc.attend_cache(q, pool.cache, *pool.where)
        assert torch.isfinite(out).all() and ((out - 3e38).abs() < 1e33).all()


def test_strides_and_alignment():
    """A pool with slots outermost, one whose rows are no whole pieces, queries of
    a fused projection."""
    for dt in TYPES:
        for rows in ([1, 2], [80, 33]):
            pool = Pool(32, dt, "plain", rows, [100, 333], 2, 64, 16)
            q = pool.queries(33, 4)
            want = dc.attend_cache(q, pool.cache, *pool.where)
            far = torch.empty(16, 2, pool.pages, 64, dtype=dt, device=DEV).permute(2, 0, 1, 3)
            off = torch.empty(pool.pages, 16, 2, 67, dtype=dt, device=DEV)[..., 1:65]
            far.copy_(pool.k)
            off.copy_(pool.v)
            wide = torch.zeros(sum(rows), 9, 64, dtype=dt, device=DEV)
            wide[:, 3:7] = q
            table = torch.full((2, 40), -1, dtype=torch.int32, device=DEV)[:, :pool.table.shape[1]]
            table.copy_(pool.table)
            assert torch.equal(want, dc.attend_cache(wide[:, 3:7], dc.Cache(far, pool.v), table, *pool.where[1:]))
            out = torch.zeros(sum(rows), 9, 65, dtype=dt, device=DEV)[:, 2:6, 1:]
            got = dc.attend_cache(q, dc.Cache(far, off), *pool.where, out=out)
            assert got is out
            check(out, None, pool.reference(q))


@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_codes_that_begin_anywhere(kind):
    """Pools of bytes that begin between two words, with rows as far apart."""
    for rows in ([1, 2], [80, 33]):
        for D, page in ((64, 16), (128, 64), (96, 32)):
            pool = Pool(52, torch.bfloat16, kind, rows, [100, 333], 2, D, page)
            q = pool.queries(53, 4)
            want = dc.attend_cache(q, pool.cache, *pool.where)

            def odd(t):
                last = t.shape[-1]
                raw = torch.zeros((pool.pages, page, 2, last + 3), dtype=torch.uint8, device=DEV)[..., 1:1 + last]
                raw.copy_(t.view(torch.uint8))
                return raw.view(t.dtype)
            cache = dc.Cache(*(odd(t) for t in (pool.k, pool.v, pool.ks, pool.vs)))
            assert torch.equal(want, dc.attend_cache(q, cache, *pool.where))


def test_rows_behind_the_last_and_longer_sequences_than_said():
    pool = Pool(34, torch.bfloat16, "e4m3", [2, 0, 40, 1], [50, 7, 60, 20], 2, 64, 16)
    q = pool.queries(35, 4, tail=9)
    out = torch.full_like(q, 7.0)
    dc.attend_cache(q, pool.cache, *pool.where, out=out)
    want = pool.reference(q)
    check(out, None, want)
    assert (out[43:] == 7.0).all()
    some = torch.full_like(q, 7.0)
    dc.attend_cache(q, pool.cache, *pool.where, out=some, max_rows=2)
    short = [0, 1, 42]
    ref.check(some[short], want.out[short], want.out_tol[short], "out")
    assert (some[2:42] == 7.0).all() and (some[43:] == 7.0).all()
    for most in (40, 41, 1000):
        assert torch.equal(out, dc.attend_cache(q, pool.cache, *pool.where, out=torch.full_like(q, 7.0), max_rows=most))


def test_calls_without_work():
    pool = Pool(36, torch.bfloat16, "e2m1", [1], [9], 1, 64, 8)
    none = torch.empty((0, 1), dtype=torch.int32, device=DEV)
    zero = torch.empty(0, dtype=torch.int32, device=DEV)
    empty = torch.empty((0, 1, 64), dtype=torch.bfloat16, device=DEV)
    assert dc.attend_cache(empty, pool.cache, none, zero).shape == (0, 1, 64)
    assert dc.attend_cache(empty, pool.cache, *pool.where[:2], ints([0, 0])).shape == (0, 1, 64)
    dc.cache_write(pool.cache, empty, empty, none, zero)
    assert dc.cache_read(pool.cache, 0, none, zero)[0].shape == (0, 1, 64)
    q = pool.queries(1, 2)
    narrow = torch.empty((1, 0), dtype=torch.int32, device=DEV)      # no table, no tokens
    assert (dc.attend_cache(q, pool.cache, narrow, pool.where[1]) == 0).all()
    assert (dc.cache_read(pool.cache, 1, narrow, pool.where[1])[0] == 0).all()


def test_offsets_that_fall_or_pass_the_rows():
    """Taken as 0 .. N, none where they fall; nothing outside the tensors is read
    or written."""
    pool = Pool(37, torch.bfloat16, "e4m3", [2, 3, 2], [20, 30, 10], 2, 64, 8)
    q = pool.queries(38, 4)
    out = torch.full_like(q, 7.0)
    dc.attend_cache(q, pool.cache, *pool.where[:2], ints([5, 2, 4, 99]), out=out)
    same = dc.attend_cache(q, pool.cache, *pool.where[:2], ints([2, 2, 4, 7]), out=torch.full_like(q, 7.0))
    assert torch.equal(out, same) and (out[:2] == 7.0).all()


def test_offsets_past_32_bits():
    """Pages past 2^32 bytes and 2^31 elements, and slots far apart."""
    dt, D, page = torch.bfloat16, 128, 16
    g = torch.Generator(device=DEV).manual_seed(40)
    stride = 1 << 26
    for rows in ([1], [40]):
        raw = torch.empty(40 * stride, dtype=dt, device=DEV)     # 5.4 GB
        k = raw.as_strided((40, page, 2, D), (stride, 2 * D, D, 1))
        v = raw.as_strided((40, page, 2, D), (stride, 2 * D, D, 1), 1 << 20)
        for t in (k, v):
            t.copy_(torch.randn(40, page, 2, D, generator=g, device=DEV))
        table = torch.arange(39, -1, -1, device=DEV, dtype=torch.int32)[None]
        q = torch.randn(rows[0], 4, D, generator=g, device=DEV).to(dt)
        n = ints([40 * page - 5])
        near = dc.Cache(k.contiguous(), v.contiguous())
        assert torch.equal(dc.attend_cache(q, dc.Cache(k, v), table, n), dc.attend_cache(q, near, table, n))
        new = torch.randn(rows[0], 2, D, generator=g, device=DEV).to(dt)
        dc.cache_write(dc.Cache(k, v), new, new, table, n)
        assert torch.equal(dc.cache_read(dc.Cache(k, v), rows[0], table, n)[0], new)
        del raw, k, v
        slots = torch.empty(page << 27, dtype=dt, device=DEV).as_strided((40, page, 2, D), (2 * D, 1 << 27, D, 1))
        slots.copy_(near.k)
        assert torch.equal(dc.attend_cache(q, dc.Cache(slots, near.v), table, n),
                           dc.attend_cache(q, near, table, n))


# ---------------------------------------------------------------------------
# calls beside one another
# ---------------------------------------------------------------------------
def step(pool, q, k, v):
    dc.cache_write(pool.cache, k, v, *pool.where)
    out, lse = dc.attend_cache(q, pool.cache, *pool.where, left=100, sinks=2, return_lse=True)
    back = dc.cache_read(pool.cache, q.shape[0], *pool.where, dtype=pool.dt)
    return (out, lse) + back


def inputs(pool, seed, Hq):
    g = torch.Generator().manual_seed(seed)
    n = sum(pool.rows)
    return tuple(torch.randn(n, h, pool.D, generator=g).to(pool.dt).to(DEV) for h in (Hq, pool.Hkv, pool.Hkv))


SETS = [([1, 1, 1], [900, 1, 70]), ([1, 90, 4], [400, 200, 33])]


@pytest.mark.parametrize("rows, lengths", SETS)
def test_equal_calls_give_equal_bits(rows, lengths):
    pool = Pool(41, torch.bfloat16, "e4m3", rows, lengths, 2, 128, 32)
    new = inputs(pool, 42, 8)
    first = step(pool, *new)
    for _ in range(10):
        for a, b in zip(first, step(pool, *new)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows, lengths", SETS)
def test_another_stream(rows, lengths):
    pool = Pool(43, torch.float16, "e2m1", rows, lengths, 2, 128, 32)
    new = inputs(pool, 44, 8)
    want = step(pool, *new)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(pool, *new)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows, lengths", SETS)
def test_two_graphs(rows, lengths):
    """Two captured steps, replayed on new rows, lengths, offsets and tables."""
    pools = [Pool(45, torch.bfloat16, "e4m3", rows, lengths, 2, 128, 32),
             Pool(46, torch.bfloat16, "plain", rows, lengths, 2, 64, 16)]
    new = [inputs(p, 47, 8) for p in pools]
    for p, x in zip(pools, new):
        step(p, *x)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for p, x in zip(pools, new):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(p, *x))
        graphs.append(graph)
    for seed in (48, 49, 50):
        for p, x in zip(pools, new):
            for old, t in zip(x, inputs(p, seed, 8)):
                old.copy_(t)
            # one token fewer each, where there are some; the chunk's rows move on
            p.where[1].copy_(ints([max(1, n - (seed - 47)) for n in lengths]))
            if seed == 50:
                p.where[2].copy_(ints([0, 1, min(20, sum(rows) - 1), sum(rows)]))
            p.where[0].copy_(p.where[0].roll(1, 1) if seed == 49 else p.where[0])
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for p, x, out in zip(pools, new, outs):
            for a, b in zip(out, step(p, *x)):
                assert torch.equal(a, b)


@pytest.mark.parametrize("kind", KINDS)
def test_a_cache_that_grows(kind):
    """A prompt in chunks, then token by token, against attention over the values
    that the cache stands for."""
    dt, page, H, D = torch.bfloat16, 16, 2, 64
    cache = dc.Cache.new(12, page, H, D, dt if kind == "plain" else kind, device=DEV)
    assert cache.pages == 12 and cache.dim == D
    table = torch.tensor([[5, 2, 9, 0, 7], [1, 11, 3, 4, 10]], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(51)
    have = [0, 0]
    for rows in ([30, 7], [0, 25], [1, 1], [1, 1], [3, 1], [40, 1]):
        n = sum(rows)
        q, k, v = (torch.randn(n, h, D, generator=g).to(dt).to(DEV) for h in (4, H, H))
        have = [a + r for a, r in zip(have, rows)]
        where = (table, ints(have), ints([0, rows[0], n]))
        dc.cache_write(cache, k, v, *where)
        out = dc.attend_cache(q, cache, *where)
        all_rows = sum(have)
        dk, dv = dc.cache_read(cache, all_rows, table, ints(have), ints([0, have[0], all_rows]), dtype=dt)
        at = 0
        for b, r in enumerate(rows):
            if r:
                lo = have[0] * b
                r_ = ref.Attend(q[at:at + r][None], dk[lo:lo + have[b]][None], dv[lo:lo + have[b]][None])
                ref.check(out[at:at + r], r_.out[0], r_.out_tol[0], "out")
                same = dc.attend(q[at:at + r][None], dk[lo:lo + have[b]][None], dv[lo:lo + have[b]][None])[0]
                ref.check(out[at:at + r], same.cpu().double(), 2 * r_.out_tol[0], "beside attend")
            at += r


def test_example_serves_in_pages():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_block
    block = token_block.TokenBlock()
    g = torch.Generator().manual_seed(60)
    with torch.no_grad():
        x = block.tokens(torch.rand((3, 3, 16, 16), generator=g).to(DEV))
        whole = block(x).float()
        for prompt in (1, 100, x.shape[1]):
            # bf16 outputs of order 1 to 4: both ways round each of five steps once
            assert (whole - block.serve_in_pages(x, prompt=prompt).float()).abs().max() <= 5 * 4 * 2.0 ** -8
        # and over codes as over the values that they stand for
        for kind in ("e4m3", "e2m1"):
            out = block.serve_in_pages(x, kind=kind)
            assert out.shape == whole.shape and torch.isfinite(out).all()


# ---------------------------------------------------------------------------
# the LDS-poisoning build, and refusals of the binding
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", [([1, 1, 1], [900, 65, 300], 8, 2, 128, 64, dict(left=200, sinks=3)),
                                  ([1, 1], [1, 500], 4, 4, 64, 16, dict()),
                                  ([130, 1, 5], [300, 260, 90], 4, 2, 64, 24, dict(left=70, sinks=2)),
                                  ([200, 33], [1500, 33], 6, 2, 96, 64, dict()),
                                  ([2, 90], [700, 120], 2, 1, 256, 32, dict()),
                                  ([40], [40], 2, 1, 32, 5, dict(left=7))], ids=str)
def test_attention_with_poisoned_lds(monkeypatch, case, kind, dt):
    path = os.path.join(os.path.dirname(dc.dconv.LIB_PATH), "libdconv_poison.so")
    if not os.path.exists(path):
        pytest.fail("libdconv_poison.so is not built (paper_2212_00404_amd/build.py builds it)")
    rows, lengths, Hq, Hkv, D, page, how = case
    pool = Pool(61, dt, kind, rows, lengths, Hkv, D, page)
    monkeypatch.setattr(dc.dconv, "_lib", dc.load(path))
    compare(pool, Hq, **how)


def test_binding_refusals():
    pool = Pool(62, torch.bfloat16, "plain", [2, 1], [20, 9], 2, 64, 8)
    table, lengths, offsets = pool.where
    c, k = pool.cache, torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=DEV)
    e4 = Pool(63, torch.bfloat16, "e4m3", [1], [9], 2, 64, 8)
    for bad in (lambda: dc.Cache(pool.k, pool.v[:1]), lambda: dc.Cache(pool.k, pool.v.half()),
                lambda: dc.Cache(pool.k, pool.v, pool.k, pool.k), lambda: dc.Cache(e4.k, e4.v),
                lambda: dc.Cache(e4.k, e4.v, e4.ks.view(torch.uint8), e4.vs), lambda: dc.Cache(pool.k[0], pool.v[0]),
                lambda: dc.Cache(e4.k, e4.v, e4.ks[..., :1], e4.vs), lambda: dc.Cache(pool.k[:0], pool.v[:0]),
                lambda: dc.Cache(pool.k[..., ::2], pool.v[..., ::2]), lambda: dc.Cache(pool.k.double(), pool.v.double()),
                lambda: dc.cache_write(c, k, k[:2], table, lengths, offsets),
                lambda: dc.cache_write(c, k.float(), k.float(), table, lengths, offsets),
                lambda: dc.cache_write(c, k[..., :32], k[..., :32], table, lengths, offsets),
                lambda: dc.cache_write(c, k[:, :1], k[:, :1], table, lengths, offsets),
                lambda: dc.cache_write(c, k, k, table.long(), lengths, offsets),
                lambda: dc.cache_write(c, k, k, table[0], lengths, offsets),
                lambda: dc.cache_write(c, k, k, table, lengths[:1], offsets),
                lambda: dc.cache_write(c, k, k, table, lengths, offsets[:2]),
                lambda: dc.cache_write(c, k, k, table, lengths), lambda: dc.cache_write(c, k, k, table.cpu(), lengths, offsets),
                lambda: dc.cache_write(c, k.cpu(), k, table, lengths, offsets),
                lambda: dc.cache_read(c, 3, table, lengths, offsets, dtype=torch.float32),
                lambda: dc.cache_read(e4.cache, 1, *e4.where, dtype=torch.float64),
                lambda: dc.cache_read(c, 3, table, lengths, offsets, out=(k[:2], k[:2])),
                lambda: dc.attend_cache(q.half(), c, table, lengths, offsets),
                lambda: dc.attend_cache(q[:, :3], c, table, lengths, offsets),
                lambda: dc.attend_cache(q[..., :32], c, table, lengths, offsets),
                lambda: dc.attend_cache(q[None], c, table, lengths, offsets),
                lambda: dc.attend_cache(q, c, table, lengths, offsets, left=-2),
                lambda: dc.attend_cache(q, c, table, lengths, offsets, sinks=-1),
                lambda: dc.attend_cache(q, c, table, lengths, offsets, max_rows=0),
                lambda: dc.attend_cache(q, c, table, lengths, offsets, left=1 << 31),
                lambda: dc.attend_cache(q, c, table, lengths, offsets, out=q[:2]),
                lambda: dc.attend_cache(q.double(), e4.cache, *e4.where),
                lambda: dc.attend_cache(q, c, table, lengths)):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros((2, 4, 1, 288), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(RuntimeError, match="-5"):
        dc.attend_cache(torch.zeros((2, 1, 288), dtype=torch.bfloat16, device=DEV), dc.Cache(wide, wide), table, lengths)
    with pytest.raises(RuntimeError, match="-2"):
        dc.attend_cache(q, c, table, lengths, offsets, scale=math.inf)
