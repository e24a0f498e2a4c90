"""GPU: keys of very small weight in fp16.  Attention's probabilities are fp16
operands; a key that weighs 2^-25 of the row's largest counts as much as its weight
says, as there may be very many of them."""
import math

import pytest
import torch

import cache_ref as cref
import paper_2212_00404_amd as dc
import token_ref as ref

pytestmark = pytest.mark.gpu
DEV, DT, D = "cuda", torch.float16, 64
KEYS = 100000
EVERY = 288     # nine tiles of 32 keys, so that every wave of four comes by a large one


def keys_and_values(scores):
    """Keys whose scores with a query of 8 in its first element are 8 * the first
    element; large ones have values of 0, the others of about 100."""
    g = torch.Generator().manual_seed(70)
    k = torch.zeros(KEYS, 1, D)
    k[:, 0, 0] = scores
    v = 100.0 + torch.randn(KEYS, 1, D, generator=g)
    v[::EVERY] = 0.0
    return k.to(DT), v.to(DT)


def far():
    k = torch.zeros(KEYS)
    k[::EVERY] = 16.0
    # e^-(8 * 16 * scale) = 2^-25.5: less than half of fp16's smallest step
    return k, 25.5 * math.log(2.0) / 128


def queries(rows, seed=71):
    g = torch.Generator().manual_seed(seed)
    q = torch.zeros(rows, 2, D)
    q[..., 0] = 8.0
    q[..., 1:] = torch.randn(rows, 2, D - 1, generator=g)   # meets zeros
    return q.to(DT)


def wanted(q, k, v, scale):
    """The definition in 64 bits with the bound of ``attend``, to which a probability's
    rounding where fp16 is subnormal is added: half its smallest step, 2^-25, where the
    row's largest (as the kernel has seen it) is 2^10 or more, so 2^-35 of that, for
    each value; divided by the sum in which the largest is 1."""
    a = ref.Attend(q[None], k[None], v[None], scale=scale)
    s = (q.double() @ k[:, 0].double().T) * scale
    see = a.see[0][:, None]
    s = s.masked_fill(~see, -math.inf)
    total = torch.exp(s - s.amax(-1, keepdim=True)).sum(-1)
    size = torch.einsum("rn,nd->rd", a.see[0].double(), v[:, 0].double().abs())
    return a.out[0], a.out_tol[0] + 2.0 ** -35 * size[:, None] / total[..., None], a.lse[0].T, a.lse_tol[0].T


def check(out, lse, q, k, v, scale):
    o, tol, l, ltol = wanted(q, k, v, scale)
    ref.check(out, o, tol, "out")
    ref.check(lse, l, ltol, "lse")


def paged(kind, k, v, page=64):
    """The same tokens as a cache, and the values that it stands for."""
    pages = -(-KEYS // page)
    cache = dc.Cache.new(pages, page, 1, D, DT if kind == "plain" else kind, device=DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    n = torch.tensor([KEYS], dtype=torch.int32, device=DEV)
    dc.cache_write(cache, k.to(DEV), v.to(DEV), table, n)
    k, v = (t.cpu() for t in dc.cache_read(cache, KEYS, table, n, dtype=DT))
    return cache, table, n, k, v


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("kind", ["plain", "e4m3", "e2m1"])
def test_many_far_keys_of_a_cache(kind, rows):
    scores, scale = far()
    cache, table, n, k, v = paged(kind, *keys_and_values(scores))
    assert torch.equal(k[:, 0, 0].float(), scores)      # the same in every format
    q = queries(rows)
    out, lse = dc.attend_cache(q.to(DEV), cache, table, n, scale=scale, return_lse=True)
    check(out, lse, q, k, v, scale)


@pytest.mark.parametrize("rows", [1, 150])
def test_many_far_keys(rows):
    scores, scale = far()
    k, v = keys_and_values(scores)
    q = queries(rows)
    out, lse = dc.attend(q[None].to(DEV), k[None].to(DEV), v[None].to(DEV), scale=scale, return_lse=True)
    check(out[0], lse[0].T, q, k, v, scale)


@pytest.mark.parametrize("step", [0.6, 3.9, 7.9])
@pytest.mark.parametrize("rows", [1, 40])
def test_scores_that_rise(rows, step):
    """Each tile's largest a few powers of two over the one before: the base lags as
    far as it may, and follows."""
    tile = torch.arange(KEYS) // 32 % 40
    scores = tile.float()
    scale = step * math.log(2.0) / 8
    cache, table, n, k, v = paged("plain", *keys_and_values(scores))
    q = queries(rows)
    out, lse = dc.attend_cache(q.to(DEV), cache, table, n, scale=scale, return_lse=True)
    check(out, lse, q, k, v, scale)
    out, lse = dc.attend(q[None].to(DEV), k[None].to(DEV), v[None].to(DEV), scale=scale, return_lse=True)
    check(out[0], lse[0].T, q, k, v, scale)
