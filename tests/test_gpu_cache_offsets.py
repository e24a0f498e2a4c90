"""GPU: offsets that fall somewhere.  Sequence b has the rows offsets[b] ..
offsets[b + 1] - 1, none where they fall, for writing, reading and attention alike."""
import pytest
import torch

import cache_ref as cref
import paper_2212_00404_amd as dc
import token_ref as ref
from test_gpu_cache import DEV, KINDS, Pool, ints

pytestmark = pytest.mark.gpu
LENGTHS = [20, 30, 10, 17]


def ranges(offsets, N):
    """Rows of each sequence, from the definition."""
    clip = (lambda x: min(max(x, 0), N))
    return [range(clip(a), max(clip(a), clip(b))) for a, b in zip(offsets, offsets[1:])]


def owners(offsets, N):
    """For each row the sequences that have it."""
    own = [[] for _ in range(N)]
    for b, rows in enumerate(ranges(offsets, N)):
        for r in rows:
            own[r].append(b)
    return own


def places(pool, lengths, offsets, N):
    """For each row (page, slot), None for a row of no sequence or of several."""
    at = [None] * N
    for r, own in enumerate(owners(offsets, N)):
        if len(own) == 1:
            rows = ranges(offsets, N)[own[0]]
            i = lengths[own[0]] - len(rows) + (r - rows.start)
            at[r] = (int(pool.table[own[0], i // pool.page]), i % pool.page)
    return at


def check_moves(pool, lengths, offsets, N):
    g = torch.Generator().manual_seed(81)
    k, v = (torch.randn(N, pool.Hkv, pool.D, generator=g).to(pool.dt) for _ in range(2))
    where = (*pool.where[:2], ints(offsets))
    own, at = owners(offsets, N), places(pool, lengths, offsets, N)
    raw = (lambda t: t.cpu().contiguous().view(torch.uint8))
    before = raw(pool.k).clone()
    dc.cache_write(pool.cache, k.to(DEV), v.to(DEV), *where)
    out = tuple(torch.full((N, pool.Hkv, pool.D), 7.0, dtype=pool.dt, device=DEV) for _ in range(2))
    dc.cache_read(pool.cache, N, *where, out=out)
    free = torch.ones(before.shape[:2], dtype=torch.bool)
    for b, rows in enumerate(ranges(offsets, N)):
        for t in range(len(rows)):
            i = lengths[b] - len(rows) + t
            free[pool.table[b, i // pool.page], i % pool.page] = False
    assert torch.equal(raw(pool.k)[free], before[free])
    for x, o, kept, scale in zip((k, v), out, (pool.k, pool.v), (pool.ks, pool.vs)):
        want = x.double()
        if pool.kind != "plain":
            code, s, _ = cref.encode(x, pool.kind)
            want = cref.decode(cref.stored(code, pool.kind), s.view(cref.SCALE), pool.kind)
        dense = cref.decode(kept, scale, pool.kind)
        for r in range(N):
            if not own[r]:
                assert (o[r] == 7.0).all(), r
            elif at[r] is not None:
                assert torch.equal(dense[at[r]], want[r]), r
                assert torch.equal(o[r].cpu().double(), want[r]), r


# offsets of up to four sequences, rows
FALLING = [
    ([4, 6, 0, 3], 7),
    ([5, 7, 0, 3, 5], 7),
    ([5, 2, 4, 99], 7),
    ([-3, 2, 1, 4], 7),
    ([7, 7, 0, 0, 7], 7),
    ([3, 0, 0, 0, 2], 9),
    ([0, 5, 3, 8], 8),          # rows 3 and 4 are of two sequences
    ([6, 8, 2, 5, 1], 8),
    ([9, 5, 3, 1, 0], 9),       # none has rows
]


@pytest.mark.parametrize("offsets, N", FALLING, ids=str)
@pytest.mark.parametrize("kind", KINDS)
def test_moves(kind, offsets, N):
    lengths = LENGTHS[:len(offsets) - 1]
    pool = Pool(80, torch.bfloat16, kind, [0] * len(lengths), lengths, 2, 64, 8)
    check_moves(pool, lengths, offsets, N)


@pytest.mark.parametrize("offsets, N", FALLING, ids=str)
@pytest.mark.parametrize("kind", KINDS)
def test_attention(kind, offsets, N):
    lengths = LENGTHS[:len(offsets) - 1]
    pool = Pool(82, torch.bfloat16, kind, [0] * len(lengths), lengths, 2, 64, 8)
    g = torch.Generator().manual_seed(83)
    q = torch.randn(N, 4, 64, generator=g).to(pool.dt)
    out = torch.full(q.shape, 7.0, dtype=pool.dt, device=DEV)
    dc.attend_cache(q.to(DEV), pool.cache, *pool.where[:2], ints(offsets), out=out)
    own, out = owners(offsets, N), out.cpu()
    for b, rows in enumerate(ranges(offsets, N)):
        mine = [0] * len(lengths)
        mine[b] = len(rows)
        pool.rows = mine
        want = pool.reference(q[rows.start:rows.stop])
        for t, r in enumerate(rows):
            if len(own[r]) == 1:
                ref.check(out[r], want.out[t], want.out_tol[t], "row %d" % r)
    for r in range(N):
        assert own[r] or (out[r] == 7.0).all(), r


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("spare", [0, 40])
def test_more_sequences_than_lds_holds(kind, spare):
    """700 sequences: the upper rows are of the first 300, the lower ones of the
    others, and some behind them of none."""
    count = [(b * 5) % 3 for b in range(700)]
    count[299] = 0                     # falls
    half = sum(count[300:])
    offsets = [half]
    for b in range(299):
        offsets.append(offsets[-1] + count[b])
    N = offsets[-1] + spare
    offsets.append(0)
    for b in range(300, 700):
        offsets.append(offsets[-1] + count[b])
    assert offsets[-1] == half and len(offsets) == 701
    lengths = [c + (b * 31) % 20 for b, c in enumerate(count)]
    pool = Pool(84, torch.bfloat16, kind, [0] * 700, lengths, 1, 32, 8)
    check_moves(pool, lengths, offsets, N)
