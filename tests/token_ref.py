"""Plain 64-bit forms (torch on the CPU, dense) of the operators over tokens,
with the sums that the tests' error bounds are made of."""
import math

import torch

# unit roundoff: half the distance from 1 to the next value
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def visible(B, Tq, Tk, left, right, sinks, lengths=None, starts=None):
    """[B, Tq, Tk]: which keys each query sees."""
    n = torch.full((B,), Tk) if lengths is None else lengths.cpu().long().clamp(0, Tk)
    s = n - Tq if starts is None else starts.cpu().long()
    i = (s[:, None] + torch.arange(Tq))[:, :, None]
    j = torch.arange(Tk)[None, None]
    see = (j < n[:, None, None]) & (i >= 0)
    if right >= 0:
        see &= j <= i + right
    if left >= 0:
        see &= (j >= i - left) | (j < sinks)
    return see


class Attend:
    """The definition on 64-bit copies: out, lse, dq, dk, dv, and a bound on the
    error of each for a kernel that keeps sums and statistics in 32 bits and
    rounds probabilities, their gradients and the result to the tensors' type.

    What the bounds are made of: products of a row lose at most D roundings of
    the sum of magnitudes (2^-24 each), which the exponential turns into a
    relative error of a probability; a rounding of probabilities is relative to
    each of them; out, as read by the backward pass, is rounded, which moves
    delta.  Twice that is allowed (the running rescaling, exp itself)."""

    def __init__(self, q, k, v, left=-1, right=0, sinks=0, scale=None, lengths=None, starts=None,
                 dout=None):
        dt = q.dtype
        u, e32 = UNIT[dt], 2.0 ** -24
        up = u if dt != torch.float32 else 0.0
        q, k, v = (t.cpu().double() for t in (q, k, v))
        B, Tq, Hq, D = q.shape
        Tk, Hkv = k.shape[1:3]
        G = Hq // Hkv
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        self.see = see = visible(B, Tq, Tk, left, right, sinks, lengths, starts)
        hid = ~see[:, None]                                           # B, 1, Tq, Tk
        Q = q.permute(0, 2, 1, 3)
        K, V = (t.permute(0, 2, 1, 3).repeat_interleave(G, 1) for t in (k, v))
        # values that no query of the batch may see are taken out (they may be NaN)
        alive = see.any(1)[:, None, :, None]
        K, V = K.masked_fill(~alive, 0.0), V.masked_fill(~alive, 0.0)
        s = (Q @ K.transpose(2, 3) * scale).masked_fill(hid, -math.inf)
        self.empty = ~see.any(2)[:, None].expand(B, Hq, Tq)
        lse = torch.logsumexp(s, -1)
        p = torch.exp(s - lse[..., None]).masked_fill(hid, 0.0)
        smag = (Q.abs() @ K.abs().transpose(2, 3) * abs(scale)).masked_fill(hid, 0.0).amax(-1)
        # relative error of a probability
        ep = 2 * (D + 8) * e32 * (smag + 1)
        self.out = (p @ V).permute(0, 2, 1, 3)
        A = p @ V.abs()
        self.lse = lse
        self.lse_tol = 2 * (ep + 2 ** -20)
        back = (lambda t: t.permute(0, 2, 1, 3))
        self.out_tol = 2 * (u * self.out.abs() + back((up + ep[..., None] + 4 * e32) * A)) + TINY[dt]
        if dout is None:
            return
        g = dout.cpu().double().permute(0, 2, 1, 3)
        O = p @ V
        dp = g @ V.transpose(2, 3)
        delta = (g * O).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        over = (lambda t: t.reshape(B, Hkv, G, Tk, D).sum(2).permute(0, 2, 1, 3))
        self.dq = back(ds @ K) * scale
        self.dk = over(ds.transpose(2, 3) @ Q) * scale
        self.dv = over(p.transpose(2, 3) @ g)
        gv = g.abs() @ V.abs().transpose(2, 3)
        go = (g.abs() * (O.abs() * u + A * (ep[..., None] + up))).sum(-1, keepdim=True)
        eds = p * ((2 * up + ep[..., None]) * (dp - delta).abs() + (D + 8) * e32 * (gv + delta.abs()) + go)
        pv = p * (up + ep[..., None])
        a = abs(scale)
        self.dq_tol = 2 * (u * self.dq.abs() + back(eds @ K.abs()) * a) + TINY[dt]
        self.dk_tol = 2 * (u * self.dk.abs() + over(eds.transpose(2, 3) @ Q.abs()) * a) + TINY[dt]
        self.dv_tol = 2 * (u * self.dv.abs() + over(pv.transpose(2, 3) @ g.abs())) + TINY[dt]


def rotate(x, positions, freq, axis, adjacent=False, inverse=False):
    """The rotation in 64 bits (the fp32 inputs are taken as they are)."""
    R, axes = freq.shape[0], positions.shape[0]
    x = x.cpu().double()
    if positions.dim() == 2:
        positions = positions[:, None].expand(-1, x.shape[0], -1)
    a = axis.cpu().long()
    ok = (a >= 0) & (a < axes)
    ang = positions.cpu().double()[a.clamp(0, axes - 1)].permute(1, 2, 0) * freq.cpu().double()
    ang = torch.where(ok, ang, 0.0)[:, :, None]
    cos, sin = torch.cos(ang), torch.sin(ang) * (-1 if inverse else 1)
    y = x.clone()
    iu = torch.arange(R) * 2 if adjacent else torch.arange(R)
    iw = iu + (1 if adjacent else R)
    u, w = x[..., iu], x[..., iw]
    y[..., iu] = u * cos - w * sin
    y[..., iw] = u * sin + w * cos
    return y


def rotate_tol(x, y, R, adjacent):
    """Two products and a sum in fp32 with sin and cos good to a few units, then
    one rounding: u |y| + 8 * 2^-24 (|u| + |w|), each pair's magnitudes."""
    dt = x.dtype
    x = x.cpu().double().abs()
    m = torch.zeros_like(x)
    iu = torch.arange(R) * 2 if adjacent else torch.arange(R)
    iw = iu + (1 if adjacent else R)
    m[..., iu] = m[..., iw] = x[..., iu] + x[..., iw]
    return 1.01 * UNIT[dt] * y.abs() + 8 * 2.0 ** -24 * m + TINY[dt]


def norm(z, kind, eps):
    if kind == "layer":
        z = z - z.mean(-1, keepdim=True)
    return z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)


def join(branch, x, norm_kind="rms", post=False, post_weight=None, gate=None, pre_weight=None,
         pre_bias=None, residual_scale=1.0, branch_scale=1.0, eps=1e-6, pre=True):
    """h and y in 64 bits; differentiable."""
    per = (lambda v: v[:, None] if v.dim() == 2 else v)
    h = residual_scale * x
    if branch is not None:
        p = branch
        if post:
            p = norm(p, norm_kind, eps)
            if post_weight is not None:
                p = p * post_weight
        h = h + branch_scale * (p if gate is None else p * per(gate))
    if not pre:
        return h, None
    y = norm(h, norm_kind, eps)
    if pre_weight is not None:
        y = y * per(pre_weight)
    if pre_bias is not None:
        y = y + per(pre_bias)
    return h, y


def check(got, want, tol, what):
    """|got - want| <= tol everywhere (and nothing but finite values)."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), "%s: %d values are not finite" % (what, (~torch.isfinite(got)).sum())
    over = (got - want).abs() - tol
    assert (over <= 0).all(), "%s: %d of %d outside, worst: off by %g where %g is allowed" % (
        what, (over > 0).sum(), over.numel(), (got - want).abs().flatten()[over.argmax()],
        (tol + torch.zeros_like(want)).flatten()[over.argmax()])
