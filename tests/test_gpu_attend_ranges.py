"""GPU: attention on values far from order 1."""
import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref
from test_gpu_attend import TYPE_IDS, TYPES, compare, make

pytestmark = pytest.mark.gpu
DEV = "cuda"


# (B, Tq, Tk, Hq, Hkv, D, window): the kernels that walk keys, that divide keys over
# workgroups of 128, 64 and 32, and that divide the rows over the first keys
GRADS = [
    (1, 1024, 1024, 2, 1, 64, dict()),
    (1, 300, 300, 4, 2, 128, dict(left=60)),
    (1, 400, 400, 2, 2, 80, dict(left=30, sinks=3)),
    (11, 300, 300, 8, 8, 40, dict(left=5, sinks=2)),
    (11, 150, 150, 8, 8, 32, dict(left=5, right=5, sinks=2)),
]
GRAD_IDS = [str(c[:6]) for c in GRADS]


# (size of dout, of the queries, of the keys).  The scores of the first three are one
# another's; larger queries make dk larger beside the probabilities' gradients, larger
# keys dq, so that it is inside the type's range where they are far below it.
SIZES = [(1e-3, 1.0, 1.0), (1e-5, 64.0, 1 / 64), (1e-5, 1 / 64, 64.0), (5e3, 0.25, 0.25)]


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("case", GRADS, ids=GRAD_IDS)
def test_gradients_of_any_size(case, size, dt):
    """The gradient is linear in dout, its error relative to dout's size: also where
    the probabilities' gradients are below the type's smallest value, or past its
    largest."""
    B, Tq, Tk, Hq, Hkv, D, how = case
    q, k, v, dout = make(31, dt, B, Tq, Tk, Hq, Hkv, D)
    compare(q * size[1], k * size[2], v, (dout.float() * size[0]).to(dt), **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("order", ["growing", "shrinking"])
@pytest.mark.parametrize("case", GRADS, ids=GRAD_IDS)
def test_gradients_of_mixed_size(case, order, dt):
    """dout and values whose size changes along the sequence, from 2^-16 to 2^4 and
    from 2^-8 to 2^4: what a row or a key is the sum of changes its size on the way."""
    B, Tq, Tk, Hq, Hkv, D, how = case
    q, k, v, dout = make(33, dt, B, Tq, Tk, Hq, Hkv, D)

    def along(t, lo, hi):
        e = torch.linspace(lo, hi, t.shape[1], device=DEV).round()
        if order == "shrinking":
            e = e.flip(0)
        return (t.float() * torch.exp2(e)[None, :, None, None]).to(dt)
    compare(q * 16, k / 16, along(v, -8, 4), along(dout, -16, 4), **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", [(1, 200, 200, 2, 1, 64, dict(left=20)), (1, 1, 300, 4, 1, 64, dict()),
                                  (2, 3, 2000, 2, 2, 40, dict()), (1, 1, 5, 1, 1, 128, dict()),
                                  (1, 70, 70, 2, 2, 200, dict())], ids=str)
def test_values_at_the_end_of_the_range(case, dt):
    """Equal scores over values of the type's largest and lowest: their mean, though
    their sum is past the range; one sign in the first half of a head, both in turn
    in the second.  Within a row the weights are one number, so that the mean is as
    good as fp32 (the definition's value rounded once, and one unit of fp32 for the
    weight)."""
    B, Tq, Tk, Hq, Hkv, D, how = case
    big = torch.finfo(dt).max
    q = torch.zeros((B, Tq, Hq, D), dtype=dt, device=DEV)
    k = torch.ones((B, Tk, Hkv, D), dtype=dt, device=DEV)
    v = torch.full((B, Tk, Hkv, D), big, dtype=dt, device=DEV)
    v[..., ::2] = -big
    v[:, ::2, :, D // 2:] *= -1
    out, lse = dc.attend(q, k, v, return_lse=True, **how)
    r = ref.Attend(q, k, v, **how)
    tol = ref.UNIT[dt] * r.out.abs() + 2 * ref.UNIT[torch.float32] * big
    ref.check(out, r.out, tol, "out")
    ref.check(lse, r.lse, r.lse_tol, "lse")
    one = dc.attend(q, k, torch.full_like(v, big), **how)
    assert (one == big).all()
