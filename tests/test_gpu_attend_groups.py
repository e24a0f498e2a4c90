"""GPU: attention's gradient where there are keys enough that a workgroup takes 128 or
64 of them (elsewhere 32): batches times key heads times keys / 128, or / 64, of 256
workgroups or more."""
import math
import os

import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref
from test_gpu_attend import TYPE_IDS, TYPES, compare, ints, make, run_both

pytestmark = pytest.mark.gpu
DEV = "cuda"
POISON = os.path.join(os.path.dirname(dc.dconv.LIB_PATH), "libdconv_poison.so")

# (B, Tq, Tk, Hq, Hkv, D, window): keys per workgroup, and whether the first keys have
# workgroups of their own (more than twice as many queries see them as a tile)
GROUPS = [
    (16, 130, 130, 16, 8, 64, dict(left=30, right=30, sinks=2)),      # 128
    (11, 300, 300, 16, 8, 40, dict(left=5, sinks=2)),                 # 128, first
    (16, 200, 200, 8, 8, 32, dict()),                                 # 128
    (11, 300, 300, 8, 8, 64, dict(left=9, right=3, sinks=37)),        # 128, first
    (8, 270, 500, 24, 8, 64, dict(left=100, sinks=1)),                # 128, three heads share keys
    (16, 127, 127, 16, 8, 64, dict(left=20)),                         # 64
    (11, 150, 150, 16, 8, 40, dict(left=5, right=5, sinks=2)),        # 64, first
    (16, 100, 100, 8, 8, 20, dict(right=-1)),                         # 64
    (16, 127, 127, 8, 8, 128, dict(left=40, sinks=3)),                # 64
    (16, 129, 129, 8, 8, 72, dict(left=40, sinks=3)),                 # 128
]
IDS = [str(c[:6]) for c in GROUPS]


def lengths_of(B, Tk):
    return [max(0, Tk - (b * 41) % (Tk + 20)) for b in range(B)]


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", GROUPS, ids=IDS)
def test_many_keys(case, dt):
    B, Tq, Tk, Hq, Hkv, D, how = case
    compare(*make(41, dt, B, Tq, Tk, Hq, Hkv, D, fused=Tq == Tk), **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", GROUPS, ids=IDS)
def test_many_keys_of_different_lengths_off_their_boundaries(case, dt):
    """Padded sequences of lengths down to 0, and rows of an odd pitch that begin on one
    element's boundary."""
    B, Tq, Tk, Hq, Hkv, D, how = case

    def pitch(t):
        big = torch.full((*t.shape[:3], D + 3), math.nan, dtype=dt, device=DEV)
        big[..., 1:1 + D] = t
        return big[..., 1:1 + D]
    args = [pitch(t) for t in make(42, dt, B, Tq, Tk, Hq, Hkv, D)]
    compare(*args, lengths=lengths_of(B, Tk), starts=[0] * B, **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("junk", [math.nan, math.inf], ids=str)
@pytest.mark.parametrize("case", GROUPS, ids=IDS)
def test_many_keys_with_junk_where_nothing_looks(case, junk, dt):
    B, Tq, Tk, Hq, Hkv, D, how = case
    q, k, v, dout = make(43, dt, B, Tq, Tk, Hq, Hkv, D)
    lengths = lengths_of(B, Tk)
    see = ref.visible(B, Tq, Tk, how.get("left", -1), how.get("right", 0), how.get("sinks", 0),
                      ints(lengths)).any(1).to(DEV)
    assert not see.all()
    clean = run_both(q, k, v, dout, lengths, **how)
    k[~see], v[~see] = junk, junk
    for a, b in zip(clean, run_both(q, k, v, dout, lengths, **how)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", [GROUPS[0], GROUPS[1], GROUPS[5], GROUPS[6]], ids=[IDS[i] for i in (0, 1, 5, 6)])
def test_nan_among_many_keys(case, dt):
    """One value of NaN: what does not see it, and what does not see what does, is what
    the definition is without it."""
    B, Tq, Tk, Hq, Hkv, D, how = case
    q, k, v, dout = make(44, dt, B, Tq, Tk, Hq, Hkv, D)
    at = Tk // 2
    see = ref.visible(B, Tq, Tk, how.get("left", -1), how.get("right", 0), how.get("sinks", 0))
    r = ref.Attend(q, k, v, dout=dout, **how)
    v[:, at] = math.nan
    out, _, dq, dk, dv = run_both(q, k, v, dout, **how)
    rows = see[0, :, at]
    keys = see[0][rows].any(0)
    assert rows.any() and not rows.all() and not keys.all()
    for name, got, hit in (("out", out, rows), ("dq", dq, rows), ("dk", dk, keys)):
        assert got[:, hit.to(DEV)].isnan().all(), name
        ref.check(got[:, ~hit.to(DEV)], getattr(r, name)[:, ~hit], getattr(r, name + "_tol")[:, ~hit], name)
    ref.check(dv, r.dv, r.dv_tol, "dv")


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", GROUPS, ids=IDS)
def test_many_keys_with_poisoned_lds(monkeypatch, case, dt):
    if not os.path.exists(POISON):
        pytest.fail("libdconv_poison.so is not built (paper_2212_00404_amd/build.py builds it)")
    monkeypatch.setattr(dc.dconv, "_lib", dc.load(POISON))
    B, Tq, Tk, Hq, Hkv, D, how = case
    compare(*make(45, dt, B, Tq, Tk, Hq, Hkv, D), **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
def test_equal_calls_of_many_keys_give_equal_bits(dt):
    for case in (GROUPS[1], GROUPS[6]):
        B, Tq, Tk, Hq, Hkv, D, how = case
        args = make(46, dt, B, Tq, Tk, Hq, Hkv, D)
        first = run_both(*args, **how)
        for _ in range(3):
            for a, b in zip(first, run_both(*args, **how)):
                assert torch.equal(a, b)
