"""GPU: windowed attention and its gradient against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]
TYPE_IDS = ["f32", "f16", "bf16"]


def make(seed, dt, B, Tq, Tk, Hq, Hkv, D, fused=False):
    g = torch.Generator().manual_seed(seed)
    def normal(*s):
        return torch.randn(s, generator=g).to(dt).to(DEV)
    if fused:
        qkv = normal(B, Tq, Hq + 2 * Hkv, D)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        q, k, v = normal(B, Tq, Hq, D), normal(B, Tk, Hkv, D), normal(B, Tk, Hkv, D)
    return q, k, v, normal(B, Tq, Hq, D)


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def run_both(q, k, v, dout, lengths=None, starts=None, **how):
    kw = dict(lengths=ints(lengths), starts=ints(starts), **how)
    out, lse = dc.attend(q, k, v, return_lse=True, **kw)
    grads = dc.attend_backward(dout, q, k, v, out, lse, **kw)
    torch.cuda.synchronize()
    return (out, lse) + grads


def compare(q, k, v, dout, lengths=None, starts=None, **how):
    out, lse, dq, dk, dv = run_both(q, k, v, dout, lengths, starts, **how)
    r = ref.Attend(q, k, v, dout=dout, lengths=ints(lengths), starts=ints(starts), **how)
    ref.check(out, r.out, r.out_tol, "out")
    lse = lse.cpu().double()
    assert (lse[r.empty] == -math.inf).all()
    ref.check(torch.where(r.empty, 0.0, lse), torch.where(r.empty, 0.0, r.lse), r.lse_tol, "lse")
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(got, getattr(r, name), getattr(r, name + "_tol"), name)
    return out, dq, dk, dv


# (B, Tq, Tk, Hq, Hkv, D, window): one key to several tiles, odd everything,
# every head size the kernels pad to, shared heads of 1, 2, 3, 4, 7
WHOLE = [
    (1, 1, 1, 1, 1, 1, dict()),
    (1, 2, 2, 2, 1, 3, dict()),
    (2, 33, 33, 4, 2, 32, dict(left=7)),
    (1, 65, 65, 3, 1, 40, dict(left=16, sinks=2)),
    (2, 127, 127, 4, 4, 64, dict(left=31, right=31, sinks=1)),
    (1, 197, 197, 7, 1, 64, dict(left=40, sinks=5)),
    (1, 300, 300, 4, 1, 72, dict(left=63, sinks=40)),
    (2, 129, 129, 6, 2, 80, dict(left=64, right=5)),
    (1, 256, 256, 2, 2, 96, dict(right=-1)),
    (1, 515, 515, 4, 1, 128, dict(left=130, sinks=4)),
    (1, 385, 385, 8, 2, 128, dict(left=0, sinks=1)),
    (1, 140, 140, 2, 1, 33, dict(left=50, sinks=3)),
    (1, 90, 90, 2, 2, 200, dict(left=20, sinks=3)),
    (1, 70, 70, 2, 1, 256, dict()),
    (1, 700, 700, 2, 1, 64, dict(left=100, right=0, sinks=70)),
]


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", WHOLE, ids=[str(c[:6]) for c in WHOLE])
def test_whole_sequences(case, dt):
    B, Tq, Tk, Hq, Hkv, D, how = case
    compare(*make(1, dt, B, Tq, Tk, Hq, Hkv, D, fused=True), **how)


# (B, Tq, Tk, Hq, Hkv, D, lengths, window): new tokens over a cache
TOKENS = [
    (1, 1, 1, 1, 1, 64, None, dict()),
    (1, 1, 196, 8, 8, 64, None, dict(left=63, sinks=1)),
    (3, 1, 700, 8, 2, 128, [700, 1, 333], dict(left=255, sinks=4)),
    (2, 1, 4000, 4, 1, 80, [4000, 2500], dict(left=2047, sinks=4)),
    (2, 5, 300, 7, 1, 64, [3, 300], dict(left=100, sinks=2)),
    (4, 1, 130, 2, 2, 40, [0, 130, 64, 65], dict()),
    (1, 17, 1000, 4, 2, 128, None, dict(left=-1)),
    (1, 3, 2000, 16, 1, 72, None, dict(left=999, sinks=8)),
    (2, 1, 500, 4, 1, 256, [500, 77], dict(left=200, sinks=1)),
]


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("case", TOKENS, ids=[str(c[:6]) for c in TOKENS])
def test_new_tokens_over_a_cache(case, dt):
    B, Tq, Tk, Hq, Hkv, D, lengths, how = case
    compare(*make(2, dt, B, Tq, Tk, Hq, Hkv, D), lengths=lengths, **how)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
def test_rows_that_see_nothing(dt):
    """Padded batches: queries past a short sequence's end see nothing once the
    window has left it; a sequence of length 0 has no row that sees anything; a
    query before position 0 sees nothing."""
    q, k, v, dout = make(3, dt, 4, 150, 150, 4, 2, 64)
    how = dict(left=20, lengths=[150, 60, 0, 150], starts=[0, 0, 0, -30])
    out, dq, dk, dv = compare(q, k, v, dout, **how)
    assert (out[1, 81:] == 0).all() and (dq[1, 81:] == 0).all()
    assert (out[2] == 0).all() and (dk[2] == 0).all() and (dv[2] == 0).all()
    assert (out[3, :30] == 0).all()
    assert (dk[1, 60:] == 0).all()


def test_no_keys_and_no_queries():
    q, k, v, dout = make(4, torch.float32, 2, 5, 0, 2, 1, 16)
    out, lse, dq, dk, dv = run_both(q, k, v, dout)
    assert (out == 0).all() and (lse == -math.inf).all() and (dq == 0).all() and dk.numel() == 0
    q, k, v, dout = make(4, torch.float32, 2, 0, 6, 2, 1, 16)
    out, lse, dq, dk, dv = run_both(q, k, v, dout)
    assert out.numel() == 0 and (dk == 0).all() and (dv == 0).all()
    q, k, v, dout = make(4, torch.float32, 0, 3, 3, 2, 1, 16)
    assert run_both(q, k, v, dout)[0].numel() == 0


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_does_not_matter(dt, junk):
    """NaN and infinities in keys and values past a sequence's end, between the
    first keys and the window, and in tiles that other queries see."""
    B, Tq, Tk, Hq, Hkv, D = 2, 40, 400, 4, 2, 64
    q, k, v, dout = make(5, dt, B, Tq, Tk, Hq, Hkv, D)
    lengths, how = [400, 211], dict(left=60, sinks=3)
    see = ref.visible(B, Tq, Tk, lengths=ints(lengths), right=0, **how).any(1).to(DEV)
    clean = run_both(q, k, v, dout, lengths, **how)
    k2, v2 = k.clone(), v.clone()
    k2[~see], v2[~see] = junk, junk
    got = run_both(q, k2, v2, dout, lengths, **how)
    for a, b in zip(clean, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("at", [0, 30, 100])
def test_nan_reaches_exactly_the_queries_that_see_it(dt, at):
    """One key and value of NaN in the middle of the tiles: the queries that see
    it are NaN, the others are what they are without it, in the gradient too."""
    B, T, Hq, Hkv, D = 1, 200, 2, 1, 64
    q, k, v, dout = make(6, dt, B, T, T, Hq, Hkv, D)
    how = dict(left=25, sinks=2)
    see = ref.visible(B, T, T, right=0, **how)[0, :, at].to(DEV)
    clean = run_both(q, k, v, dout, **how)
    v2 = v.clone()
    v2[:, at] = math.nan
    got = run_both(q, k, v2, dout, **how)
    r = ref.Attend(q, k, v, dout=dout, **how)
    assert got[0][:, see].isnan().all() and not got[0][:, ~see].isnan().any()
    ref.check(got[0][:, ~see], r.out[:, ~see.cpu()], r.out_tol[:, ~see.cpu()], "out")
    assert got[2][:, see].isnan().all()
    ref.check(got[2][:, ~see], r.dq[:, ~see.cpu()], r.dq_tol[:, ~see.cpu()], "dq")
    # dv does not read v; its probabilities do not either
    ref.check(got[4], r.dv, r.dv_tol, "dv")
    seen_by_them = ref.visible(B, T, T, right=0, **how)[0][see.cpu()].any(0).to(DEV)
    assert got[3][:, seen_by_them].isnan().all()
    ref.check(got[3][:, ~seen_by_them], r.dk[:, ~seen_by_them.cpu()], r.dk_tol[:, ~seen_by_them.cpu()], "dk")


@pytest.mark.parametrize("dt", TYPES, ids=TYPE_IDS)
def test_lowest_values_and_large_scores(dt):
    """Keys of the type's lowest value (a mask by value) get no weight beside
    ordinary ones; scores of thousands do not overflow."""
    q, k, v, dout = make(7, dt, 1, 50, 50, 2, 2, 32)
    low = torch.finfo(dt).min
    q = q.abs() + 0.1
    k2 = k.clone()
    k2[:, 1::2] = low
    out, lse = dc.attend(q, k2, v, return_lse=True, scale=1.0)
    qs, ks = q.cpu().double(), k2.cpu().double()
    see = ref.visible(1, 50, 50, -1, 0, 0)[:, None]
    s = (qs.permute(0, 2, 1, 3) @ ks.permute(0, 2, 3, 1)).masked_fill(~see, -math.inf)
    want = (torch.softmax(s, -1) @ v.cpu().double().permute(0, 2, 1, 3)).permute(0, 2, 1, 3)
    tol = 4 * ref.UNIT[dt] * v.abs().max().item() + 1e-4
    ref.check(out, want, tol, "out")
    big = compare(q, k, v, dout, scale=100.0) if dt == torch.float32 else None
    assert big is None or torch.isfinite(big[0]).all()


def test_strides_and_alignment():
    """Heads first in memory, rows off 16-byte boundaries, an odd row pitch, a
    broadcast batch and an output with strides of its own: the bits of the
    contiguous call."""
    for dt in TYPES:
        q, k, v, dout = make(8, dt, 2, 90, 90, 4, 2, 64)
        k, v = k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1)
        how = dict(left=30, sinks=2)
        want = run_both(q, k, v, dout, **how)

        def pitch(t, lead, extra):
            big = torch.full((*t.shape[:3], t.shape[3] + extra), float("nan"), dtype=dt, device=DEV)
            big[..., lead:lead + t.shape[3]] = t
            return big[..., lead:lead + t.shape[3]]
        first = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v, dout)]
        odd = [pitch(t, 1, 3) for t in (q, k, v, dout)]
        even = [pitch(t, 8, 16) for t in (q, k, v, dout)]
        for args in (first, odd, even):
            got = run_both(*args, **how)
            r = ref.Attend(q, k, v, dout=dout, **how)
            for name, i in (("out", 0), ("dq", 2), ("dk", 3), ("dv", 4)):
                ref.check(got[i], getattr(r, name), getattr(r, name + "_tol"), name)
        o = torch.full((2, 4, 90, 70), float("nan"), dtype=dt, device=DEV).permute(0, 2, 1, 3)[..., 3:67]
        got = dc.attend(q, k, v, out=o, **how)
        assert got is o and torch.equal(o, want[0])


def test_offsets_past_32_bits():
    """A cache whose last sequence starts past 2^32 bytes and 2^31 elements."""
    B, Tk, H, D = 3, 90000, 64, 128          # 2.2e9 elements in bf16
    k = torch.empty((B, Tk, H, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = torch.Generator(device=DEV).manual_seed(9)
    n = 100
    k[2, Tk - n:] = torch.randn((n, H, D), generator=g, device=DEV).bfloat16()
    v[2, Tk - n:] = torch.randn((n, H, D), generator=g, device=DEV).bfloat16()
    q = torch.randn((B, 1, H, D), generator=g, device=DEV).bfloat16()
    out = dc.attend(q, k, v, left=n - 1, lengths=ints([0, 0, Tk]))
    r = ref.Attend(q[2:], k[2:, Tk - n:].contiguous(), v[2:, Tk - n:].contiguous(), left=n - 1)
    ref.check(out[2:], r.out, r.out_tol, "out")
    assert (out[:2] == 0).all()


@pytest.mark.parametrize("what", ["queries", "keys"])
def test_rows_far_apart(what):
    """Tokens 16 MB apart: a tile of rows spans more than 2^32 bytes."""
    dt, T, D = torch.bfloat16, 300, 64
    q, k, v, dout = make(16, dt, 1, T, T, 1, 1, D)
    far = torch.empty((1, T, 1, 1 << 23), dtype=dt, device=DEV)[..., :D]
    far.copy_(q if what == "queries" else k)
    args = (far, k, v, dout) if what == "queries" else (q, far, v, dout)
    want, got = run_both(q, k, v, dout, left=200), run_both(*args, left=200)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_equal_calls_give_equal_bits():
    q, k, v, dout = make(10, torch.bfloat16, 2, 333, 333, 8, 2, 64)
    how = dict(left=90, sinks=5)
    first = run_both(q, k, v, dout, **how)
    for _ in range(10):
        for a, b in zip(first, run_both(q, k, v, dout, **how)):
            assert torch.equal(a, b)


def test_another_stream():
    q, k, v, dout = make(11, torch.bfloat16, 2, 200, 200, 4, 2, 64)
    want = run_both(q, k, v, dout, left=50, sinks=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run_both(q, k, v, dout, left=50, sinks=1)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_in_a_graph():
    """A captured forward and backward pass, replayed on new inputs."""
    q, k, v, dout = make(12, torch.bfloat16, 1, 150, 150, 4, 2, 64)
    qt, kt, vt, _ = make(13, torch.bfloat16, 2, 1, 900, 4, 1, 64)
    how = dict(left=40, sinks=2)
    run_both(q, k, v, dout, **how)
    dc.attend(qt, kt, vt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = dc.attend(q, k, v, return_lse=True, **how)
        grads = dc.attend_backward(dout, q, k, v, out, lse, **how)
        one = dc.attend(qt, kt, vt)
    for seed in (20, 21, 22):
        for old, new in zip((q, k, v, dout, qt, kt, vt),
                            make(seed, torch.bfloat16, 1, 150, 150, 4, 2, 64) +
                            make(seed, torch.bfloat16, 2, 1, 900, 4, 1, 64)[:3]):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = run_both(q, k, v, dout, **how)
        for a, b in zip(want, (out, lse) + grads):
            assert torch.equal(a, b)
        assert torch.equal(one, dc.attend(qt, kt, vt))


@pytest.mark.parametrize("Hq, Hkv, D, how", [(4, 2, 16, dict(left=9, sinks=2)), (2, 2, 40, dict(left=5, right=5)),
                                             (3, 1, 64, dict())])
def test_gradients_against_differences(Hq, Hkv, D, how):
    """fp32: along random directions the gradient is what the 64-bit definition
    changes by (central differences; third derivatives leave 1e-8, fp32 sums of
    a few thousand terms 1e-5)."""
    q, k, v, dout = make(14, torch.float32, 1, 37, 37, Hq, Hkv, D)
    _, _, dq, dk, dv = run_both(q, k, v, dout, **how)
    g = torch.Generator().manual_seed(15)
    base = [t.cpu().double() for t in (q, k, v)]
    for i, grad in enumerate((dq, dk, dv)):
        d = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        eps = 1e-4

        def f(sign):
            args = list(base)
            args[i] = args[i] + sign * eps * d
            see = ref.visible(1, 37, 37, how.get("left", -1), how.get("right", 0), how.get("sinks", 0))[:, None]
            G = Hq // Hkv
            Q = args[0].permute(0, 2, 1, 3)
            K, V = (t.permute(0, 2, 1, 3).repeat_interleave(G, 1) for t in args[1:])
            s = (Q @ K.transpose(2, 3) / math.sqrt(D)).masked_fill(~see, -math.inf)
            return ((torch.softmax(s, -1) @ V).permute(0, 2, 1, 3) * dout.cpu().double()).sum()
        want = (f(1) - f(-1)) / (2 * eps)
        got = (grad.cpu().double() * d).sum()
        size = (grad.cpu().double() * d).abs().sum()
        assert abs(got - want) <= 1e-5 * size + 1e-6, (i, got, want)
