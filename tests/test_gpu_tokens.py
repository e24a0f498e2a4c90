"""GPU: the operators over tokens together (the example), their refusals in the
binding, and the build whose LDS starts as NaN."""
import math
import os
import sys

import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
POISON = os.path.join(os.path.dirname(dc.dconv.LIB_PATH), "libdconv_poison.so")

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_example_trains_and_serves():
    import token_block
    losses, off = token_block.main()
    assert losses[-1] < 0.5 * losses[0], losses
    # bf16 outputs of order 1 to 4: both ways round each of five steps once
    assert off <= 5 * 4 * 2.0 ** -8


def test_block_gradient_against_differences():
    """The whole block in fp32: the gradient of a loss along a random direction."""
    import token_block
    block = token_block.TokenBlock(channels=16, rows=4, cols=5, Hq=2, Hkv=1, head=8, left=7, dtype=torch.float32)
    g = torch.Generator().manual_seed(2)
    images = torch.rand((2, 3, 6, 7), generator=g).cuda()
    w = torch.randn((2, 21, 16), generator=g).cuda()

    def loss():
        return (block(block.tokens(images)) * w).double().sum()
    params = [p for p in block.parameters if p is not block.out]
    grads = torch.autograd.grad(loss(), params)
    for p, grad in zip(params, grads):
        d = torch.randn(p.shape, generator=g).cuda()
        with torch.no_grad():
            eps = 1e-2
            p += eps * d
            up = loss()
            p -= 2 * eps * d
            down = loss()
            p += eps * d
        want, terms = (up - down) / (2 * eps), grad.double() * d.double()
        # fp32 sums of 672 terms of order 1 to 10: 2e-5 each way, over 2 eps; third
        # derivatives of order 10 times eps^2
        assert abs(want - terms.sum()) <= 5e-3 + 2e-3 * terms.abs().sum(), (tuple(p.shape), want, terms.sum())


def poisoned(monkeypatch):
    if not os.path.exists(POISON):
        pytest.fail("libdconv_poison.so is not built (paper_2212_00404_amd/build.py builds it)")
    monkeypatch.setattr(dc.dconv, "_lib", dc.load(POISON))


# whole tiles and parts of them, divided keys and rows, aligned rows and others
POISONED = [(1, 300, 300, 4, 2, 64, dict(left=70, sinks=3)), (1, 1, 900, 8, 2, 128, dict(left=500, sinks=4)),
            (2, 33, 33, 3, 1, 80, dict(left=9)), (1, 7, 150, 2, 2, 33, dict()), (8, 256, 256, 16, 8, 40, dict(left=50)),
            (16, 130, 130, 8, 8, 128, dict(left=30, right=30, sinks=2)), (1, 40, 40, 2, 1, 200, dict())]


@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", POISONED, ids=[str(c[:6]) for c in POISONED])
def test_attend_with_poisoned_lds(monkeypatch, case, dt):
    poisoned(monkeypatch)
    B, Tq, Tk, Hq, Hkv, D, how = case
    g = torch.Generator().manual_seed(3)
    q, k, v, dout = (torch.randn(s, generator=g).to(dt).to(DEV)
                     for s in ((B, Tq, Hq, D), (B, Tk, Hkv, D), (B, Tk, Hkv, D), (B, Tq, Hq, D)))
    out, lse = dc.attend(q, k, v, return_lse=True, **how)
    grads = dc.attend_backward(dout, q, k, v, out, lse, **how)
    r = ref.Attend(q, k, v, dout=dout, **how)
    ref.check(out, r.out, r.out_tol, "out")
    for name, got in zip(("dq", "dk", "dv"), grads):
        ref.check(got, getattr(r, name), getattr(r, name + "_tol"), name)


@pytest.mark.parametrize("size", [(2, 5, 64), (3, 40, 1000), (1, 9, 4096), (2, 300, 2048), (1, 3, 16384)])
def test_join_with_poisoned_lds(monkeypatch, size):
    B, T, D = size
    g = torch.Generator().manual_seed(4)
    b, x, dh, dy = (torch.randn(size, generator=g).to(DEV) for _ in range(4))
    vec = {n: torch.rand(D, generator=g).to(DEV) + 0.5 for n in ("post_weight", "gate", "pre_weight", "pre_bias")}

    def both():
        h, y, stats = dc.join(b, x, norm="layer", post=True, return_stats=True, **vec)
        grads = dc.join_backward(dh, dy, b, x, stats, norm="layer", post=True, **vec)
        return [h, y, stats] + [grads[n] for n in sorted(grads)]
    want = both()
    poisoned(monkeypatch)
    for a, c in zip(want, both()):
        assert torch.equal(a, c)


def test_binding_refusals():
    q = torch.zeros((2, 5, 4, 16), device=DEV)
    k = torch.zeros((2, 7, 2, 16), device=DEV)
    n = torch.zeros(2, dtype=torch.int32, device=DEV)
    for bad in (lambda: dc.attend(q, k.half(), k), lambda: dc.attend(q, k, k[:, :6]),
                lambda: dc.attend(q, k[:1], k[:1]), lambda: dc.attend(q[:, :, :3], k, k),
                lambda: dc.attend(q, k.transpose(1, 3), k.transpose(1, 3)), lambda: dc.attend(q, k, k, left=-2),
                lambda: dc.attend(q, k, k, sinks=-1), lambda: dc.attend(q, k, k, lengths=n.long()),
                lambda: dc.attend(q, k, k, lengths=n[:1]), lambda: dc.attend(q, k, k, starts=n.cpu()),
                lambda: dc.attend(q, k, k, out=q[:, :4]), lambda: dc.attend(q, k, k.cpu()),
                lambda: dc.attend_backward(q[:, :3], q, k, k, q, torch.zeros((2, 4, 5), device=DEV)),
                lambda: dc.attend_backward(q, q, k, k, q, torch.zeros((2, 5, 4), device=DEV)),
                lambda: dc.attend(torch.zeros((2, 5, 4), device=DEV), k, k)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError, match="-5"):
        dc.attend(torch.zeros((1, 1, 1, 300), device=DEV), *[torch.zeros((1, 1, 1, 300), device=DEV)] * 2)
    with pytest.raises(RuntimeError, match="-2"):
        dc.attend(q, k, k, scale=math.inf)
    at, freq, axis = torch.zeros((1, 2, 5), device=DEV), torch.ones(8, device=DEV), n.new_zeros(8)
    for bad in (lambda: dc.rotate(q, at.double(), freq, axis), lambda: dc.rotate(q, at[:, :, :4], freq, axis),
                lambda: dc.rotate(q, at, freq, axis[:7]), lambda: dc.rotate(q, at, freq, axis.long()),
                lambda: dc.rotate(q, at, torch.ones(9, device=DEV), n.new_zeros(9)),
                lambda: dc.rotate(q, at[:0], freq, axis), lambda: dc.rotate(q, at, freq, axis, out=q.half())):
        with pytest.raises(ValueError):
            bad()
    x, w = torch.zeros((2, 3, 8), device=DEV), torch.ones(8, device=DEV)
    for bad in (lambda: dc.join(x[:1], x), lambda: dc.join(x, x, norm="batch"), lambda: dc.join(x, x, gate=w[:7]),
                lambda: dc.join(x, x, post_weight=w), lambda: dc.join(None, x, gate=w),
                lambda: dc.join(None, x, pre=False), lambda: dc.join(x, x, pre=False, pre_weight=w),
                lambda: dc.join(x, x, gate=w.half()), lambda: dc.join(x.half(), x.half(), gate=w, pre_weight=w.half()),
                lambda: dc.join(x, x, gate=torch.ones((3, 8), device=DEV)),
                lambda: dc.join_backward(x, x, x, x, torch.zeros((2, 3, 3), device=DEV))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("option", [dict(left=1 << 31), dict(right=1 << 40), dict(sinks=1 << 31), dict(left=3.0)],
                         ids=str)
def test_options_past_32_bits_are_refused_by_the_binding(option):
    q = torch.zeros((1, 2, 1, 16), device=DEV)
    with pytest.raises(ValueError):
        dc.attend(q, q, q, **option)
