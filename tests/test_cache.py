"""A cache in pages without a GPU: refusals of the C ABI and of the binding, the
packed structs, workspace queries, and the plain forms that the GPU tests compare
with."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

import cache_ref as cref
import paper_2212_00404_amd as dc
from paper_2212_00404_amd import cache as binding
from paper_2212_00404_amd import dconv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000      # never dereferenced: validation comes first


def cache_struct(pages=5, page_size=16, Hkv=2, D=64, format=0, dtype=2):
    s = (page_size * Hkv * D, D, page_size * D)
    return binding._CACHE.pack(pages, page_size, Hkv, D, format, dtype, *(s * 4))


def rows_struct(B=3, N=6, width=4, dtype=2, stride=4):
    return binding._ROWS.pack(B, N, width, dtype, stride, 128, 64, 128, 64)


def attend_struct(B=3, N=6, width=4, Hq=4, dtype=2, left=-1, right=0, sinks=0, max_rows=0, scale=0.1):
    return binding._ATTEND.pack(B, N, width, Hq, dtype, left, right, sinks, max_rows, scale, 4, 256, 64, 256, 64)


def write(cache, rows, k=P, v=P, ck=P, cv=P, ks=P, vs=P, table=P, lengths=P, offsets=P):
    return dc.load().dconv_cache_write(cache, rows, k, v, ck, cv, ks, vs, table, lengths, offsets, None)


def read(cache, rows, k=P, v=P, ck=P, cv=P, ks=P, vs=P, table=P, lengths=P, offsets=P):
    return dc.load().dconv_cache_read(cache, rows, ck, cv, ks, vs, table, lengths, offsets, k, v, None)


def attend(cache, shape, q=P, ck=P, cv=P, ks=P, vs=P, table=P, lengths=P, offsets=P, out=P, lse=P, ws=P, n=1 << 40):
    return dc.load().dconv_cache_attend(cache, shape, q, ck, cv, ks, vs, table, lengths, offsets, out, lse, ws, n, None)


def workspace(cache, shape):
    n = ctypes.c_longlong(-1)
    return dc.load().dconv_cache_attend_workspace(cache, shape, ctypes.byref(n)), n.value


def test_null_pointers():
    for f in (write, read):
        for name in ("cache", "rows", "k", "v", "ck", "cv", "table", "lengths"):
            args = {"cache": cache_struct(), "rows": rows_struct(), name: None}
            assert f(**args) == dconv.ENULL, (f.__name__, name)
        for name in ("ks", "vs"):
            assert f(cache_struct(format=1), rows_struct(), **{name: None}) == dconv.ENULL
    for name in ("cache", "shape", "q", "ck", "cv", "table", "lengths", "out"):
        args = {"cache": cache_struct(), "shape": attend_struct(), name: None}
        assert attend(**args) == dconv.ENULL, name
    for name in ("ks", "vs"):
        assert attend(cache_struct(format=2), attend_struct(), **{name: None}) == dconv.ENULL
    assert dc.load().dconv_cache_attend_workspace(cache_struct(), attend_struct(), None) == dconv.ENULL


@pytest.mark.parametrize("bad", [dict(pages=0), dict(page_size=0), dict(Hkv=0), dict(D=0), dict(format=3),
                                 dict(format=-1), dict(dtype=3)], ids=str)
def test_caches_that_are_none(bad):
    assert write(cache_struct(**bad), rows_struct()) == dconv.EINVAL
    assert read(cache_struct(**bad), rows_struct()) == dconv.EINVAL
    assert attend(cache_struct(**bad), attend_struct()) == dconv.EINVAL
    assert workspace(cache_struct(**bad), attend_struct())[0] == dconv.EINVAL


@pytest.mark.parametrize("bad", [dict(B=-1), dict(N=-1), dict(width=-1), dict(dtype=5), dict(dtype=0)], ids=str)
def test_rows_that_are_none(bad):
    """(Rows of a plain cache are of its type.)"""
    assert write(cache_struct(), rows_struct(**bad)) == dconv.EINVAL
    assert read(cache_struct(), rows_struct(**bad)) == dconv.EINVAL


@pytest.mark.parametrize("bad", [dict(B=-1), dict(N=-1), dict(width=-1), dict(Hq=0), dict(Hq=3), dict(dtype=7),
                                 dict(dtype=1), dict(left=-2), dict(right=-2), dict(sinks=-1), dict(max_rows=-1),
                                 dict(scale=math.inf), dict(scale=math.nan)], ids=str)
def test_attention_refusals(bad):
    assert attend(cache_struct(), attend_struct(**bad)) == dconv.EINVAL
    assert workspace(cache_struct(), attend_struct(**bad))[0] == dconv.EINVAL


def test_rows_without_offsets_are_alike():
    for f in (write, read):
        assert f(cache_struct(), rows_struct(B=4, N=6), offsets=None) == dconv.EINVAL
        assert f(cache_struct(), rows_struct(B=0, N=6), offsets=None) == dconv.EINVAL
    assert attend(cache_struct(), attend_struct(B=4), offsets=None) == dconv.EINVAL
    assert attend(cache_struct(), attend_struct(B=0), offsets=None) == dconv.EINVAL


def test_sizes_that_are_not_supported():
    for f, s in ((write, rows_struct), (read, rows_struct), (attend, attend_struct)):
        assert f(cache_struct(D=257), s()) == dconv.EUNSUPPORTED
        assert f(cache_struct(D=80, format=1), s()) == dconv.EUNSUPPORTED
        assert f(cache_struct(D=80, format=2), s()) == dconv.EUNSUPPORTED
        assert f(cache_struct(), s(width=1 << 27)) == dconv.ERANGE           # 2^31 tokens
        assert f(cache_struct(page_size=1 << 30), s()) == dconv.ERANGE
        assert f(cache_struct(), s(B=(1 << 20) + 1)) == dconv.ERANGE
        assert f(cache_struct(Hkv=4098), s(**(dict(Hq=4098) if f is attend else {}))) == dconv.ERANGE
    assert attend(cache_struct(Hkv=1), attend_struct(N=1 << 28, Hq=8)) == dconv.ERANGE
    assert workspace(cache_struct(Hkv=1), attend_struct(N=1 << 28, Hq=8))[0] == dconv.ERANGE


def test_launches_that_do_not_fit_are_refused():
    """A launch has less than 2^32 threads."""
    small = cache_struct(Hkv=1, D=8, page_size=1 << 10)
    for f in (write, read):
        assert f(small, rows_struct(B=1, N=1 << 30, width=1 << 20)) == dconv.ERANGE


def test_calls_without_work_need_no_device():
    for f, s in ((write, rows_struct), (read, rows_struct), (attend, attend_struct)):
        assert f(cache_struct(), s(N=0), ck=None) == 0
        assert f(cache_struct(), s(B=0, N=0), lengths=None, offsets=None) == 0
    assert workspace(cache_struct(), attend_struct(N=0)) == (0, 0)


def test_workspaces():
    """Little for few rows over short tables, and bounded: two parts of each of 512
    workgroups at most, of 32 and of 128 rows."""
    assert workspace(cache_struct(), attend_struct(N=3, width=32, max_rows=1)) == (0, 0)      # 512 tokens
    sizes = [workspace(cache_struct(D=128), attend_struct(B=b, N=n, width=w))[1]
             for b, n, w in ((1, 1, 64), (1, 1, 1 << 20), (64, 64, 1 << 12), (64, 1 << 20, 1 << 20))]
    assert all(s > 0 for s in sizes)
    part = 2 * (128 + 2) * 4
    assert max(sizes) <= 512 * (32 + 128) * part + 2 * 512 * 2 * 64
    for shape in (attend_struct(width=1 << 10), attend_struct(N=600, width=1 << 10, max_rows=200)):
        rc, n = workspace(cache_struct(), shape)
        assert rc == 0 and n > 0
        assert attend(cache_struct(), shape, n=n - 1) == dconv.EWORKSPACE
        assert attend(cache_struct(), shape, ws=None) == dconv.ENULL
        assert attend(cache_struct(), shape, ws=P + 4) == dconv.EINVAL


def test_a_workspace_is_for_what_the_call_launches():
    """Rows without offsets are N / B each, whatever max_rows says: a workspace for
    fewer is refused."""
    shape = attend_struct(B=2, N=400, width=1 << 10, max_rows=1)
    n = workspace(cache_struct(), shape)[1]
    assert attend(cache_struct(), shape, offsets=None, n=n) == dconv.EWORKSPACE


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_packed_structs_are_the_headers(tmp_path):
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dconv.h"\n'
                   "int main(void) { printf(\"%zu %zu %zu %zu %zu %zu %zu\\n\", sizeof(dconv_cache),"
                   " offsetof(dconv_cache, k_stride), sizeof(dconv_cache_rows),"
                   " offsetof(dconv_cache_rows, table_stride), sizeof(dconv_cache_attend_shape),"
                   " offsetof(dconv_cache_attend_shape, scale),"
                   " offsetof(dconv_cache_attend_shape, table_stride)); return 0; }\n")
    exe = str(tmp_path / "size")
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    c, r, a = binding._CACHE.size, binding._ROWS.size, binding._ATTEND.size
    assert got == [c, c - 96, r, r - 40, a, 36, a - 40]


def test_binding_refuses_tensors_on_the_host():
    k = torch.zeros(3, 4, 2, 64)
    with pytest.raises(ValueError, match="must be on a HIP device"):
        dc.Cache(k, k)
    with pytest.raises(ValueError, match="must be a torch.Tensor"):
        dc.Cache(None, k)
    with pytest.raises(ValueError, match="got torch.float64"):
        dc.Cache(k.double(), k.double())
    with pytest.raises(ValueError, match="must be on a HIP device"):
        dc.Cache.new(3, 4, 2, 64, device="cpu")
    for kind in ("int8", torch.float64):
        with pytest.raises(ValueError, match="kind must be"):
            dc.Cache.new(3, 4, 2, 64, kind, device="cpu")
    with pytest.raises(ValueError, match="multiple of 32"):
        dc.Cache.new(3, 4, 2, 80, "e4m3", device="cpu")
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be a Cache"):
        dc.cache_read(k, 1, n[None], n)
    with pytest.raises(ValueError, match="must be a Cache"):
        dc.attend_cache(k[0], (k, k), n[None], n)
    with pytest.raises(ValueError, match=r"\[N, heads, D\]"):
        dc.cache_write(None, k, k, n[None], n)


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", ["e4m3", "e2m1"])
def test_reference_codes_are_the_nearest(kind, dt):
    """By search over all codes; and torch's own e4m3 where it has one."""
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(40, 64, generator=g) * torch.exp2(torch.randint(-9, 9, (40, 1), generator=g))).to(dt)
    x[3], x[4, :32] = 0, torch.finfo(dt).max
    code, scale, bad = cref.encode(x, kind)
    assert not bad.any()
    back = cref.decode(cref.stored(code, kind), scale.view(cref.SCALE), kind)
    s = torch.exp2(scale.double() - 127).repeat_interleave(32, -1)
    grid = torch.cat([-cref.GRID[kind], cref.GRID[kind]])
    limited = x.double().clamp(-cref.limit(kind, dt), cref.limit(kind, dt))
    best = (limited[..., None] - grid * s[..., None]).abs().amin(-1)
    assert torch.equal((limited - back).abs(), best)
    top = limited.abs().unflatten(-1, (-1, 32)).amax(-1)
    some = top > 0
    sc = torch.exp2(scale.double() - 127)
    assert (cref.LARGEST[kind] * sc >= top).all() and (cref.LARGEST[kind] * sc / 2 < top)[some].all()
    if kind == "e4m3":
        assert torch.equal((limited / s).float().to(torch.float8_e4m3fn).float().double(), back / s)


def test_reference_attention_by_loops():
    """A cache with a page that is none, a window and first keys, by loops."""
    g = torch.Generator().manual_seed(2)
    page, D = 4, 3
    k, v = (torch.randn(6, page, 2, D, generator=g) for _ in range(2))
    table = torch.tensor([[4, 9, 2], [0, 1, -1]], dtype=torch.int32)
    lengths, rows = [11, 6], [3, 2]
    q = torch.randn(5, 4, D, generator=g)
    r = cref.Attend(q, k, v, None, None, "plain", table, lengths, rows, left=3, sinks=2)
    at = 0
    for b in range(2):
        for t in range(rows[b]):
            i = lengths[b] - rows[b] + t
            for h in range(4):
                ws, vs = [], []
                for j in range(lengths[b]):
                    p = int(table[b, j // page])
                    if j <= i and (j >= i - 3 or j < 2) and 0 <= p < 6:
                        ws.append(float(q[at, h].double() @ k[p, j % page, h // 2].double()) / math.sqrt(D))
                        vs.append(v[p, j % page, h // 2].double())
                w = torch.softmax(torch.tensor(ws, dtype=torch.float64), 0)
                want = (w[:, None] * torch.stack(vs)).sum(0)
                assert (r.out[at, h] - want).abs().max() < 1e-12
                assert abs(float(r.lse[at, h]) - math.log(sum(math.exp(x) for x in ws))) < 1e-12
            at += 1
