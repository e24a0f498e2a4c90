"""GPU: rotary positions with several axes against the rotation in 64 bits."""
import math

import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
TYPE_IDS = ["f32", "f16", "bf16"]


def table(pairs, interleaved=False):
    return dc.rotary_table(pairs, interleaved=interleaved, device=DEV)


def compare(x, positions, freq, axis, **how):
    y = dc.rotate(x, positions, freq, axis, **how)
    want = ref.rotate(x, positions, freq, axis, **how)
    ref.check(y, want, ref.rotate_tol(x, want, freq.shape[0], how.get("adjacent", False)), "rotate")
    return y


# (B, T, H, D, pairs per axis): one value to odd sizes, part of a head, no pair
CASES = [(1, 1, 1, 2, (1,)), (2, 3, 1, 7, (1, 1)), (1, 5, 3, 64, (8, 12, 12)), (2, 57, 4, 128, (16, 24, 24)),
         (3, 20, 5, 72, (8, 4, 4)), (1, 33, 2, 80, (20, 20)), (8, 1, 24, 64, (32,)), (1, 7, 2, 33, (5, 5, 6)),
         (2, 6, 2, 16, ()), (1, 300, 40, 128, (64,)), (1, 4, 2, 256, (30, 30, 30, 30))]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", CASES, ids=[str(c) for c in CASES])
def test_rotation(case, dt, adjacent):
    B, T, H, D, pairs = case
    g = torch.Generator().manual_seed(1)
    x = torch.randn((B, T, H, D), generator=g).to(dt).to(DEV)
    at = (torch.rand((max(1, len(pairs)), B, T), generator=g) * 300).to(DEV)
    for inverse in (False, True):
        compare(x, at, *table(pairs, interleaved=adjacent), adjacent=adjacent, inverse=inverse)


def test_large_and_odd_positions():
    """The angle loses nothing at large, negative and fractional positions."""
    x = torch.randn((1, 8, 2, 64), device=DEV)
    at = torch.tensor([[[0.0, -1.0, 0.5, 4095.75, 65536.0, 1e6, -123456.0, 16777216.0]]], device=DEV)
    compare(x, at, *table((32,)))
    compare(x, at, torch.linspace(0.5, 7.0, 32, device=DEV), torch.zeros(32, dtype=torch.int32, device=DEV))


def test_strides_in_place_and_shared_positions():
    """Heads of a fused projection, rows off 16-byte boundaries, positions of one
    sequence for the batch, and the input as output: the values of the plain
    call."""
    freq, axis = table((8, 12, 12))
    at = dc.map_positions(2, 5, 3, device=DEV)
    for dt in TYPES:
        for lead, width in ((0, 64), (1, 67), (8, 80)):
            big = torch.randn((2, 30, 6, width), device=DEV).to(dt)
            x = big[:, :, 1:5, lead:lead + 64]
            want = compare(x.contiguous(), at[:, None].expand(3, 2, 30).contiguous(), freq, axis)
            assert torch.equal(compare(x, at, freq, axis), want)
            rest = big.clone()
            assert dc.rotate(x, at, freq, axis, out=x) is x
            assert torch.equal(x, want)
            rest[:, :, 1:5, lead:lead + 64] = want
            assert torch.equal(rest, big)      # nothing beside the heads was written


def test_there_and_back():
    """The inverse is the transpose (the gradient): <rotate(x), g> = <x, inverse(g)>,
    and it undoes the rotation."""
    freq, axis = table((8, 12, 12))
    at = dc.map_positions(2, 9, 7, device=DEV)
    x, g = torch.randn((2, 1, 126, 3, 64), device=DEV).unbind(0)
    y, back = dc.rotate(x, at, freq, axis), dc.rotate(g, at, freq, axis, inverse=True)
    a, b = (y.double() * g.double()).sum(), (x.double() * back.double()).sum()
    assert abs(a - b) <= 1e-6 * (y.double() * g.double()).abs().sum()
    assert (dc.rotate(y, at, freq, axis, inverse=True) - x).abs().max() < 2e-6


def test_gradient_against_differences():
    freq, axis = table((6, 5))
    g = torch.Generator().manual_seed(3)
    x, d, dy = (torch.randn((1, 10, 2, 30), generator=g) for _ in range(3))
    at = torch.rand((2, 10), generator=g) * 50
    def f(z):
        return (ref.rotate(z, at, freq, axis, adjacent=True) * dy.double()).sum()
    want = (f(x.double() + 1e-3 * d.double()) - f(x.double() - 1e-3 * d.double())) / 2e-3
    dx = dc.rotate(dy.to(DEV), at.to(DEV), freq, axis, adjacent=True, inverse=True).cpu().double()
    assert abs((dx * d).sum() - want) <= 1e-5 * (dx * d).abs().sum()


def test_axes_out_of_range_leave_pairs_as_they_are():
    x = torch.randn((1, 4, 1, 8), device=DEV)
    at = torch.rand((2, 4), device=DEV) * 9
    axis = torch.tensor([0, 2, -1, 1], dtype=torch.int32, device=DEV)
    y = compare(x, at, torch.ones(4, device=DEV), axis)
    assert torch.equal(y[..., [1, 2, 5, 6]], x[..., [1, 2, 5, 6]])


def test_empty_calls_and_special_values():
    freq, axis = table((4,))
    for shape in ((0, 3, 2, 8), (2, 0, 2, 8)):
        assert dc.rotate(torch.empty(shape, device=DEV), torch.empty((1,) + shape[:2], device=DEV),
                         freq, axis).shape == shape
    x = torch.ones((1, 3, 1, 12), device=DEV)
    x[0, 1, 0, 9] = math.nan                     # not rotated: copied, and nowhere else
    x[0, 2, 0, 0] = math.inf
    y = dc.rotate(x, torch.rand((1, 3), device=DEV), freq, axis)
    assert y[0, 1, 0, 9].isnan() and not y[0, 1, 0, :9].isnan().any()
    assert not y[0, 0].isnan().any() and y[0, 2, 0, 1:4].isfinite().all()


def test_offsets_past_32_bits():
    x = torch.empty((1, 3, 1, 1 << 30), dtype=torch.bfloat16, device=DEV)[..., :64]
    x.copy_(torch.randn((1, 3, 1, 64), device=DEV))
    at = torch.arange(3, device=DEV).float()[None]
    compare(x, at, *table((32,)))


def test_another_stream_and_a_graph():
    freq, axis = table((32,))
    at = torch.arange(40, device=DEV).float()[None]
    x = torch.randn((2, 40, 4, 64), device=DEV)
    want = dc.rotate(x, at, freq, axis)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = dc.rotate(x, at, freq, axis)
    torch.cuda.synchronize()
    assert torch.equal(want, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = dc.rotate(x, at, freq, axis)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, dc.rotate(x, at, freq, axis))


def test_as_many_sequences_as_are_counted():
    """2^31 - 1 of them: the workgroups' steps over them pass 32 bits.  (No pair is
    turned, the one value of each is copied.)"""
    B = (1 << 31) - 1
    x = torch.empty((B, 1, 1, 1), dtype=torch.float16, device=DEV)
    x.view(-1).copy_((torch.arange(1 << 12, device=DEV) % 2039).half().repeat(1 << 19)[:B])
    at = torch.zeros((1, 1, 1), device=DEV).expand(1, B, 1)
    none = torch.zeros(0, device=DEV)
    out = dc.rotate(x, at, none, none.int())
    assert torch.equal(out, x)
