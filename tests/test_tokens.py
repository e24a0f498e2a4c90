"""The operators over tokens without a GPU: refusals of the C ABI and of the
binding, the packed structs, workspace queries, and the 64-bit forms that the GPU
tests compare with."""
import ast
import ctypes
import inspect
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2212_00404_amd as dc
import token_ref as ref
from paper_2212_00404_amd import build, dconv, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000      # never dereferenced: validation comes first


def rotate_shape(B=2, T=3, H=4, D=64, R=32, axes=1, adjacent=0, inverse=0, dtype=0):
    return tokens._ROTATE_SHAPE.pack(B, T, H, D, R, axes, adjacent, inverse, dtype, T * H * D, H * D, D,
                                     T * H * D, H * D, D, B * T, T, 1)


def join_shape(B=2, T=3, D=64, dtype=0, vt=0, norm=0, post=1, per=0, eps=1e-6):
    return tokens._JOIN_SHAPE.pack(B, T, D, dtype, vt, norm, post, per, 1.0, 1.0, eps, *([T * D, D] * 4))


def attend_shape(B=2, Tq=5, Tk=7, Hq=4, Hkv=2, D=64, dtype=0, left=3, right=0, sinks=1, scale=0.1):
    q, k = (Tq * Hq * D, Hq * D, D), (Tk * Hkv * D, Hkv * D, D)
    return tokens._ATTEND_SHAPE.pack(B, Tq, Tk, Hq, Hkv, D, dtype, left, right, sinks, scale, *q, *k, *k, *q, *q)


def rotate(shape, x=P, pos=P, freq=P, axis=P, out=P):
    return dc.load().dconv_rotate(shape, x, pos, freq, axis, out, None)


def join(shape, branch=P, x=P, pw=P, gate=P, w=P, bias=P, h=P, y=P, stats=P):
    return dc.load().dconv_join(shape, branch, x, pw, gate, w, bias, h, y, stats, None)


def join_backward(shape, dh=P, dy=P, branch=P, x=P, pw=P, gate=P, w=P, stats=P, dbranch=P, dx=P, dpw=P,
                  dgate=P, dw=P, dbias=P, ws=P, n=1 << 40):
    return dc.load().dconv_join_backward(shape, dh, dy, branch, x, pw, gate, w, stats, dbranch, dx, dpw, dgate,
                                         dw, dbias, ws, n, None)


def attend(shape, q=P, k=P, v=P, lengths=None, starts=None, out=P, lse=P, ws=P, n=1 << 40):
    return dc.load().dconv_attend(shape, q, k, v, lengths, starts, out, lse, ws, n, None)


def attend_backward(shape, dout=P, q=P, k=P, v=P, out=P, lse=P, dq=P, dk=P, dv=P, ws=P, n=1 << 40):
    return dc.load().dconv_attend_backward(shape, dout, q, k, v, out, lse, None, None, dq, dk, dv, ws, n, None)


def test_null_pointers():
    for f, names in ((rotate, ("shape", "x", "pos", "freq", "axis", "out")), (join, ("shape", "x", "h")),
                     (join_backward, ("shape", "x", "stats", "dbranch", "dx")),
                     (attend, ("shape", "q", "k", "v", "out")),
                     (attend_backward, ("shape", "dout", "q", "k", "v", "out", "lse", "dq", "dk", "dv"))):
        good = {rotate: rotate_shape, attend: attend_shape, attend_backward: attend_shape}.get(f, join_shape)()
        for name in names:
            args = {"shape": good, name: None}
            assert f(**args) == dconv.ENULL, (f.__name__, name)
    assert join(join_shape(), h=None, y=None, branch=None) == dconv.ENULL     # nothing to write
    for name in ("pw", "gate", "w"):                                          # a gradient of a missing vector
        assert join_backward(join_shape(), **{name: None}) == dconv.ENULL


@pytest.mark.parametrize("bad", [dict(B=-1), dict(T=-1), dict(H=0), dict(D=0), dict(R=-1), dict(R=33),
                                 dict(axes=0), dict(adjacent=2), dict(inverse=-1), dict(dtype=3)])
def test_rotate_refusals(bad):
    assert rotate(rotate_shape(**bad)) == dconv.EINVAL


@pytest.mark.parametrize("bad", [dict(B=-1), dict(T=-1), dict(D=0), dict(dtype=5), dict(vt=1), dict(dtype=1, vt=2),
                                 dict(norm=2), dict(post=2), dict(per=16), dict(eps=-1.0), dict(eps=math.nan)])
def test_join_refusals(bad):
    assert join(join_shape(**bad)) == dconv.EINVAL
    assert join_backward(join_shape(**bad)) == dconv.EINVAL
    n = ctypes.c_longlong()
    assert dc.load().dconv_join_workspace(join_shape(**bad), ctypes.byref(n)) == dconv.EINVAL


@pytest.mark.parametrize("bad", [dict(B=-1), dict(Tq=-1), dict(Tk=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=3),
                                 dict(D=0), dict(dtype=-1), dict(left=-2), dict(right=-2), dict(sinks=-1),
                                 dict(scale=math.inf), dict(scale=math.nan)])
def test_attend_refusals(bad):
    assert attend(attend_shape(**bad)) == dconv.EINVAL
    assert attend_backward(attend_shape(**bad)) == dconv.EINVAL
    n = ctypes.c_longlong()
    assert dc.load().dconv_attend_workspace(attend_shape(**bad), ctypes.byref(n)) == dconv.EINVAL
    assert dc.load().dconv_attend_backward_workspace(attend_shape(**bad), ctypes.byref(n)) == dconv.EINVAL


def test_sizes_that_are_not_supported():
    assert attend(attend_shape(D=257)) == dconv.EUNSUPPORTED
    assert join(join_shape(D=16385)) == dconv.ERANGE
    assert join(join_shape(B=1 << 16, T=1 << 15)) == dconv.ERANGE
    assert attend(attend_shape(B=1 << 12, Hq=1 << 10, Tk=1 << 10)) == dconv.ERANGE
    assert rotate(rotate_shape(T=(1 << 31) - 1, H=64)) == dconv.ERANGE


def test_launches_that_do_not_fit_are_refused():
    """A launch has less than 2^32 threads."""
    assert attend(attend_shape(B=1 << 24, Tq=1, Tk=1, Hq=1, Hkv=1)) == dconv.ERANGE
    assert attend_backward(attend_shape(B=1 << 24, Tq=1, Tk=1, Hq=1, Hkv=1)) == dconv.ERANGE
    assert attend_backward(attend_shape(B=1, Tq=1, Tk=1 << 28, Hq=1, Hkv=1, D=200)) == dconv.ERANGE
    assert join(join_shape(B=1 << 22, T=1, per=1)) == dconv.ERANGE
    n = ctypes.c_longlong()
    assert dc.load().dconv_attend_workspace(attend_shape(B=1 << 24, Hq=1, Hkv=1), ctypes.byref(n)) == dconv.ERANGE


@pytest.mark.parametrize("sizes", [dict(Tq=1, Tk=(1 << 31) - 2), dict(Tq=1, Tk=(1 << 31) - (1 << 16)),
                                   dict(Tq=(1 << 31) - (1 << 16), Tk=1), dict(Tq=(1 << 28) - 100, Tk=1, Hq=8)],
                         ids=str)
def test_walks_past_32_bits_are_refused(sizes):
    """Keys and rows are counted in 32 bits by steps that end up to 2^16 past the last
    one."""
    shape = attend_shape(**{**dict(B=1, Hq=1, Hkv=1, D=1, left=-1), **sizes})
    assert attend(shape) == dconv.ERANGE
    assert attend_backward(shape) == dconv.ERANGE
    n = ctypes.c_longlong()
    assert dc.load().dconv_attend_workspace(shape, ctypes.byref(n)) == dconv.ERANGE
    assert dc.load().dconv_attend_backward_workspace(shape, ctypes.byref(n)) == dconv.ERANGE


def test_the_longest_walk_is_accepted():
    shape = attend_shape(B=1, Tq=1, Tk=(1 << 31) - 1 - (1 << 16), Hq=1, Hkv=1, D=1, left=-1)
    n = ctypes.c_longlong()
    assert dc.load().dconv_attend_workspace(shape, ctypes.byref(n)) == 0


def test_workspaces_off_their_boundary():
    assert attend(attend_shape(B=1, Tq=1, Tk=100000, left=-1), ws=P + 8) == dconv.EINVAL
    assert attend_backward(attend_shape(), ws=P + 4) == dconv.EINVAL
    assert join_backward(join_shape(B=4, T=1000), ws=P + 8) == dconv.EINVAL


def test_branch_and_gradients_that_do_not_go_together():
    assert join_backward(join_shape(), branch=None) == dconv.ENULL
    assert join_backward(join_shape(), branch=None, dbranch=None) == dconv.EINVAL
    assert join_backward(join_shape(post=0)) == dconv.EINVAL          # a gradient of post_weight without post
    assert join(join_shape(), stats=P + 4) == dconv.EINVAL            # off a 16-byte boundary


def test_workspaces():
    n = ctypes.c_longlong()
    lib = dc.load()
    assert lib.dconv_attend_workspace(attend_shape(), ctypes.byref(n)) == 0
    # one token over a long cache: the keys are divided, the parts' sums kept
    long = attend_shape(B=1, Tq=1, Tk=100000, left=-1)
    assert lib.dconv_attend_workspace(long, ctypes.byref(n)) == 0 and n.value > 0
    assert attend(long, n=n.value - 1) == dconv.EWORKSPACE
    assert attend(long, ws=None) == dconv.ENULL
    assert lib.dconv_attend_backward_workspace(attend_shape(), ctypes.byref(n)) == 0 and n.value > 0
    assert attend_backward(attend_shape(), n=n.value - 1) == dconv.EWORKSPACE
    many = join_shape(B=4, T=1000)
    assert lib.dconv_join_workspace(many, ctypes.byref(n)) == 0 and n.value > 0
    assert join_backward(many, n=n.value - 1) == dconv.EWORKSPACE
    for f in (lib.dconv_attend_workspace, lib.dconv_attend_backward_workspace):
        assert f(None, ctypes.byref(n)) == dconv.ENULL and f(attend_shape(), None) == dconv.ENULL


def test_a_workspace_is_needed_without_rows_too():
    """The gradients of vectors are written (zeros) where there are no rows, by way of
    the workspace where there are several sequences."""
    none = join_shape(B=3, T=0, per=2)
    n = ctypes.c_longlong()
    assert dc.load().dconv_join_workspace(none, ctypes.byref(n)) == 0 and n.value > 0
    assert join_backward(none, ws=None) == dconv.ENULL
    assert join_backward(none, ws=None, n=0) == dconv.ENULL


def test_as_many_rows_as_are_counted_are_divided_into_runs():
    """2^31 - 1 rows take as many runs, whose sums the workspace holds, as 2^30 do."""
    n = ctypes.c_longlong()
    sizes = []
    for T in (1 << 30, (1 << 31) - 1):
        assert dc.load().dconv_join_workspace(join_shape(B=1, T=T, D=1), ctypes.byref(n)) == 0
        sizes.append(n.value)
    assert sizes[0] > 0 and abs(sizes[1] - sizes[0]) <= sizes[0] // 100


def test_calls_without_work_need_no_device():
    assert rotate(rotate_shape(B=0), x=None, out=None) == 0
    assert rotate(rotate_shape(T=0)) == 0
    assert join(join_shape(B=0), x=None) == 0
    assert attend(attend_shape(B=0), q=None) == 0
    assert attend(attend_shape(Tq=0), q=None) == 0
    assert attend_backward(attend_shape(B=0)) == 0


def test_strerror_of_the_workspace():
    assert "workspace" in dc.strerror(dconv.EWORKSPACE)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_packed_structs_are_the_headers(tmp_path):
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dconv.h"\n'
                   "int main(void) { printf(\"%zu %zu %zu %zu %zu %zu\\n\", sizeof(dconv_rotate_shape),"
                   " offsetof(dconv_rotate_shape, x_stride), sizeof(dconv_join_shape),"
                   " offsetof(dconv_join_shape, branch_stride), sizeof(dconv_attend_shape),"
                   " offsetof(dconv_attend_shape, q_stride)); return 0; }\n")
    exe = str(tmp_path / "size")
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    r, j, a = tokens._ROTATE_SHAPE.size, tokens._JOIN_SHAPE.size, tokens._ATTEND_SHAPE.size
    assert got == [r, r - 72, j, j - 64, a, a - 120]


def test_binding_refuses_tensors_on_the_host():
    x = torch.zeros(1, 2, 2, 8)
    with pytest.raises(ValueError, match="must be on a HIP device"):
        dc.attend(x, x, x)
    with pytest.raises(ValueError, match="must be on a HIP device"):
        dc.rotate(x, torch.zeros(1, 1, 2), torch.ones(4), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="must be on a HIP device"):
        dc.join(x[0], x[0])
    with pytest.raises(ValueError, match="must be a torch.Tensor"):
        dc.attend(None, x, x)
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        dc.attend(x.double(), x, x)


def test_rotary_table_and_map_positions():
    freq, axis = dc.rotary_table((2, 3), base=100.0)
    assert axis.tolist() == [0, 0, 1, 1, 1]
    assert freq.tolist() == pytest.approx([1, 0.1, 1, 100 ** (-1 / 3), 100 ** (-2 / 3)])
    freq, axis = dc.rotary_table((2, 3, 1), interleaved=True)
    assert axis.tolist() == [0, 1, 2, 0, 1, 1]
    assert [t.numel() for t in dc.rotary_table(())] == [0, 0]
    assert dc.map_positions(2, 2, 3).tolist() == [[0] * 6 + [1] * 6, [0, 0, 0, 1, 1, 1] * 2, [0, 1, 2] * 4]


@pytest.mark.parametrize("how", [dict(), dict(left=3), dict(left=2, right=2, sinks=1), dict(right=-1), dict(left=0)])
def test_reference_attention_by_loops_and_autograd(how):
    """The 64-bit form against a loop over keys and against autograd."""
    g = torch.Generator().manual_seed(0)
    q, dout = torch.randn((2, 6, 4, 5), generator=g), torch.randn((2, 6, 4, 5), generator=g)
    k, v = torch.randn((2, 9, 2, 5), generator=g), torch.randn((2, 9, 2, 5), generator=g)
    lengths, starts = torch.tensor([9, 4]), torch.tensor([2, -1])
    r = ref.Attend(q, k, v, dout=dout, lengths=lengths, starts=starts, **how)
    left, right, sinks = how.get("left", -1), how.get("right", 0), how.get("sinks", 0)
    qd, kd, vd = (t.double().requires_grad_() for t in (q, k, v))
    rows = []
    for b in range(2):
        for t in range(6):
            i = int(starts[b]) + t
            js = [j for j in range(int(lengths[b])) if i >= 0 and (right < 0 or j <= i + right)
                  and (left < 0 or j >= i - left or j < sinks)]
            for h in range(4):
                if not js:
                    rows.append(qd.new_zeros(5))
                    continue
                s = torch.stack([(qd[b, t, h] * kd[b, j, h // 2]).sum() for j in js]) / math.sqrt(5)
                w = torch.exp(s - s.max())
                rows.append((w[:, None] * torch.stack([vd[b, j, h // 2] for j in js])).sum(0) / w.sum())
    out = torch.stack(rows).reshape(2, 6, 4, 5)
    assert torch.allclose(out, r.out, atol=1e-12)
    for want, got in zip(torch.autograd.grad((out * dout.double()).sum(), [qd, kd, vd]), (r.dq, r.dk, r.dv)):
        assert torch.allclose(want, got, atol=1e-12)


def test_reference_rotation_keeps_lengths_and_composes():
    g = torch.Generator().manual_seed(1)
    x = torch.randn((1, 4, 2, 12), generator=g)
    freq, axis = dc.rotary_table((2, 3))
    one = torch.ones((2, 4))
    for adjacent in (False, True):
        y = ref.rotate(x, one * 3, freq, axis, adjacent)
        assert torch.allclose(y.norm(dim=-1), x.double().norm(dim=-1))
        twice = ref.rotate(ref.rotate(x, one * 1.5, freq, axis, adjacent), one * 1.5, freq, axis, adjacent)
        assert torch.allclose(twice, y, atol=1e-12)
        assert torch.equal(y[..., 10:], x[..., 10:].double())
        assert torch.allclose(ref.rotate(y, one * 3, freq, axis, adjacent, inverse=True), x.double(), atol=1e-12)


@pytest.mark.skipif(shutil.which(build._hipcc()) is None, reason="needs hipcc")
@pytest.mark.parametrize("element", ["_Float16", "__bf16", "float", "float2"])
def test_the_poisoning_build_fills_lds_of_any_element(tmp_path, element):
    """Its kernels begin by writing their LDS: the code of one that only does that and
    reads it back has a write, whatever the elements' size."""
    src = tmp_path / "fill.hip"
    src.write_text('#include "internal.h"\n'
                   "extern \"C\" __global__ void fill(%s *out) {\n"
                   "  __shared__ __align__(16) %s buf[256];\n"
                   "  DCONV_POISON(dconv::poison_lds(buf, 256));\n"
                   "  out[threadIdx.x] = buf[255 - threadIdx.x];\n}\n" % (element, element))
    res = subprocess.run([build._hipcc()] + build.CFLAGS + ["-DDCONV_POISON_LDS", "--offload-device-only", "-S",
                                                            str(src), "-o", str(tmp_path / "fill.s")],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    code = (tmp_path / "fill.s").read_text()
    assert "ds_read" in code and "ds_write" in code


def test_the_readme_calls_what_there_is():
    """Its calls fit the functions' signatures, and the tables of a rotation are made on
    a device (rotate takes no others)."""
    with open(os.path.join(ROOT, "README.md"), encoding="utf-8") as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    calls = [c for b in blocks for c in ast.walk(ast.parse(b)) if isinstance(c, ast.Call)
             and isinstance(c.func, ast.Attribute) and getattr(c.func.value, "id", None) == "dc"]
    assert {"attend", "attend_backward", "rotate", "join"} <= {c.func.attr for c in calls}
    for c in calls:
        inspect.signature(getattr(dc, c.func.attr)).bind(*c.args, **{k.arg: k.value for k in c.keywords})
        if c.func.attr in ("rotary_table", "map_positions"):
            assert "device" in [k.arg for k in c.keywords], ast.unparse(c)
