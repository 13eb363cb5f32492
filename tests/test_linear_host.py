"""Refusals of the linear layers' products without a GPU: the C ABI on pointers that are never dereferenced, the Python path on tensors of
the CPU or without storage."""
import ctypes
import os
import re

import pytest
import torch

from paper_2403_16863_amd import binding, linear

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ON_CPU = not torch.cuda.is_available()


def p(x):
    return ctypes.c_void_p(x)


def m(data, stride=64):
    return linear.Rows(data, stride)


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "linear.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b((?:gemm_)?linear[a-z_0-9]*)\s*\(", text)))
    assert names == sorted(linear.SYMBOLS)
    for n in names:
        assert hasattr(linear.lib(), n) and (hasattr(linear, n) or n.endswith("_with"))     # (those are the native call path's)


# 5 rows of 64 columns (x: 5 x 64, w: 64 x 32 or 32 x 64), rows of 128 bytes
def forward(x=m(0x10000), w=m(0x20000, 32), rows_of_n=0, bias=0x30000, f32=0, res=m(0x40000), pre=m(0x50000), out=m(0x60000), act=2, M=5, N=32, K=64, dt=1,
            ws=0, bytes_=0):
    return linear.lib().gemm_linear(x, w, rows_of_n, p(bias), f32, res, pre, out, act, M, N, K, dt, p(ws), bytes_, None)


def backward(dy=m(0x10000), x=m(0x20000), w=m(0x30000, 32), rows_of_n=0, pre=m(0x40000), dx=m(0x50000), dw=m(0x60000, 32), dw_rows_of_n=0, dbias=0x70000, act=1,
             M=5, N=32, K=64, dt=0, ws=0x100000, bytes_=1 << 20):
    return linear.lib().gemm_linear_bwd(dy, x, w, rows_of_n, pre, dx, dw, dw_rows_of_n, p(dbias), act, M, N, K, dt, p(ws), bytes_, None)


NONE = m(None)


def test_forward_refuses_bad_arguments():
    for bad in (dict(x=NONE), dict(w=NONE), dict(out=NONE), dict(x=m(0x10008)), dict(out=m(0x60002)), dict(bias=0x30008), dict(res=m(0x40004)),
                dict(pre=m(0x50008)), dict(M=0), dict(M=-1), dict(N=0), dict(N=12), dict(K=0), dict(K=60), dict(dt=2), dict(dt=-1), dict(act=5), dict(act=-1),
                dict(x=m(0x10000, 56)), dict(x=m(0x10000, 68)), dict(w=m(0x20000, 24)), dict(w=m(0x20000, 32), rows_of_n=1), dict(out=m(0x60000, 0)),
                dict(out=m(0x60000, -64)), dict(ws=0x70008)):
        assert forward(**bad) == linear.LINEAR_EINVAL, bad
    for bad in (dict(N=(1 << 22) + 8, w=m(0x20000000, 1 << 23)), dict(K=(1 << 22) + 8), dict(M=(1 << 30) + 1), dict(x=m(0x10000, (1 << 22) + 8))):
        assert forward(**bad) == linear.LINEAR_EUNSUPPORTED, bad


def test_forward_refuses_outputs_over_other_memory():
    for bad in (dict(out=m(0x10000)), dict(out=m(0x10000 + 5 * 128 - 16)), dict(out=m(0x20000)), dict(out=m(0x40000, 128)), dict(out=m(0x40000 + 16)),
                dict(out=m(0x50000)), dict(pre=m(0x60000 + 32)), dict(pre=m(0x40000)), dict(pre=m(0x10000 + 64)), dict(out=m(0x30000)), dict(out=m(0x30000 - 128)),
                dict(x=m(0x10000, 128), out=m(0x10000 + 256 - 16, 128))):
        assert forward(**bad) == linear.LINEAR_EINVAL, bad


@pytest.mark.skipif(not ON_CPU, reason="the addresses are nobody's")
def test_what_is_not_refused():
    """Nothing can be launched here, so a call that passes the checks is refused by the runtime."""
    for good in (dict(), dict(res=NONE), dict(pre=NONE, bias=0), dict(out=m(0x40000)), dict(M=1, out=m(0x40000, 3), res=m(0x40000, 0)), dict(M=1, x=m(0x10000, -7)),
                 dict(x=m(0x10000, 128), out=m(0x10000 + 128, 128)), dict(x=m(0x10000, 128), out=m(0x10000 - 64, 128)), dict(rows_of_n=1, w=m(0x20000, 64))):
        assert forward(**good) == linear.LINEAR_ELAUNCH, good
    for good in (dict(), dict(dx=NONE, w=NONE), dict(dw=NONE, x=NONE), dict(dbias=0), dict(act=0, pre=NONE), dict(dx=NONE, dw=NONE, x=NONE, w=NONE),
                 dict(dw_rows_of_n=1, dw=m(0x60000, 64)), dict(act=0, dbias=0, ws=0, bytes_=0)):
        assert backward(**good) == linear.LINEAR_ELAUNCH, good


def test_backward_refuses_bad_arguments():
    for bad in (dict(dx=NONE, dw=NONE, dbias=0), dict(dy=NONE), dict(w=NONE), dict(x=NONE), dict(pre=NONE), dict(dbias=0x70008), dict(ws=0x100008), dict(act=9), dict(M=0), dict(N=4), dict(K=4), dict(dt=3), dict(dw=m(0x60000, 24)), dict(dw_rows_of_n=1),
                dict(dx=m(0x50008)), dict(dy=m(0x10000, 24))):
        assert backward(**bad) == linear.LINEAR_EINVAL, bad
    for bad in (dict(ws=0), dict(bytes_=0), dict(bytes_=16)):
        assert backward(**bad) == linear.LINEAR_ENOMEM, bad
    for bad in (dict(dx=m(0x10000)), dict(dx=m(0x20000)), dict(dx=m(0x60000)), dict(dw=m(0x20000, 32)), dict(dw=m(0x40000, 32)), dict(dbias=0x60000),
                dict(dbias=0x10000), dict(ws=0x50000 - 256), dict(ws=0x30000)):
        assert backward(**bad) == linear.LINEAR_EINVAL, bad
    for bad in (dict(M=(1 << 30) + 1), dict(N=(1 << 22) + 8), dict(K=(1 << 22) + 8)):
        assert backward(**bad) == linear.LINEAR_EUNSUPPORTED, bad


def test_memory_asked_for_by_the_call():
    """Once, with the bytes of the workspace functions, and none without a use for it."""
    if not ON_CPU:
        pytest.skip("the addresses are nobody's")
    asked = []

    def scratch(owner, n):
        asked.append((owner, n))
        return None
    fn, L = linear.SCRATCH_FN(scratch), linear.lib()
    M, N, K = 4, 64, 16384
    args = (m(0x1000000, K), m(0x2000000, N), 0, None, 0, NONE, NONE, m(0x3000000, N), 0, M, N, K, 0, fn, p(7), None)
    rc = L.gemm_linear_with(*args)
    assert asked == [(7, linear.gemm_linear_workspace(M, N, K))] and rc == linear.LINEAR_ELAUNCH
    asked.clear()
    back = (m(0x1000000, N), m(0x2000000, K), m(0x3000000, N), 0, m(0x4000000, N), m(0x5000000, K), m(0x6000000, N), 0, None, 1, M, N, K, 0, fn, None, None)
    assert L.gemm_linear_bwd_with(*back) == linear.LINEAR_ENOMEM
    assert asked == [(None, linear.gemm_linear_bwd_workspace(M, N, K, "relu", dbias=False))]
    asked.clear()
    assert L.gemm_linear_with(NONE, *args[1:]) == linear.LINEAR_EINVAL and L.gemm_linear_bwd_with(NONE, *back[1:]) == linear.LINEAR_EINVAL and not asked


def test_no_memory_is_asked_for_by_calls_that_are_refused():
    """Neither for bad arguments nor for outputs over other memory: the overlap is what the caller hears of, not the missing memory."""
    asked = []
    fn, L = linear.SCRATCH_FN(lambda owner, n: asked.append(n)), linear.lib()

    def ask(dy=m(0x10000), x=m(0x20000), w=m(0x30000, 32), pre=m(0x40000), dx=m(0x50000), dw=m(0x60000, 32), dbias=0x70000, N=32, act=1):
        return L.gemm_linear_bwd_with(dy, x, w, 0, pre, dx, dw, 0, p(dbias), act, 5, N, 64, 0, fn, None, None)
    for bad in (dict(dx=m(0x10000)), dict(dx=m(0x20000)), dict(dx=m(0x60000)), dict(dw=m(0x20000, 32)), dict(dw=m(0x40000, 32)), dict(dbias=0x60000),
                dict(dbias=0x10000), dict(dx=m(0x70000 - 16)), dict(N=12), dict(act=5), dict(pre=NONE), dict(dx=m(0x50008))):
        assert ask(**bad) == linear.LINEAR_EINVAL and not asked, bad
    assert ask() == linear.LINEAR_ENOMEM and len(asked) == 1
    for bad in (dict(out=m(0x1000000, 64)), dict(out=m(0x2000000, 64)), dict(pre=m(0x3000000, 64)), dict(res=m(0x3000000 + 16, 64))):
        t = {"out": m(0x3000000, 64), "pre": NONE, "res": NONE, **bad}
        rc = L.gemm_linear_with(m(0x1000000, 16384), m(0x2000000, 64), 0, None, 0, t["res"], t["pre"], t["out"], 0, 4, 64, 16384, 0, fn, None, None)
        assert rc == linear.LINEAR_EINVAL and len(asked) == 1, bad


def test_products_refuse_bad_arguments():
    L = linear.lib()

    def call(a=m(0x10000), b=m(0x20000), layout=0, c=m(0x30000), M=16, N=64, K=64, dt=0, tile=0, ranges=1, ws=0, bytes_=0):
        return L.linear_product(a, b, layout, c, M, N, K, dt, tile, ranges, p(ws), bytes_, None)
    for bad in (dict(layout=3), dict(layout=-1), dict(tile=-1), dict(tile=linear.linear_num_tiles()), dict(ranges=0), dict(ranges=33), dict(layout=2, M=20),
                dict(K=63), dict(N=4), dict(M=0), dict(a=NONE), dict(c=m(0x10000)), dict(dt=2), dict(ranges=2, K=4096, a=m(0x10000, 4096), b=m(0x200000))):
        assert call(**bad) == linear.LINEAR_EINVAL, bad
    with pytest.raises(linear.LinearError):
        linear.linear_choice(8, 12, 8, 0)
    with pytest.raises(linear.LinearError):
        linear.linear_choice(2 ** 40, 8, 8, 0)


def test_workspaces_by_size():
    assert linear.gemm_linear_workspace(4096, 4096, 512) == 0 and linear.gemm_linear_workspace(4, 64, 16384) > 0
    assert linear.gemm_linear_bwd_workspace(4096, 4096, 4096, dbias=False) == 0            # dz is dy
    assert linear.gemm_linear_bwd_workspace(4096, 4096, 4096, "relu", dbias=False) >= 2 * 4096 * 4096
    for bad in ((0, 8, 8), (8, 12, 8), (8, 8, 2 ** 33)):
        with pytest.raises(linear.LinearError):
            linear.gemm_linear_workspace(*bad)
        with pytest.raises(linear.LinearError):
            linear.gemm_linear_bwd_workspace(*bad)
    with pytest.raises(linear.LinearError):
        linear.gemm_linear_bwd_workspace(8, 8, 8, dx=False, dw=False, dbias=False)


def test_python_names_what_it_refuses():
    from torch._subclasses.fake_tensor import FakeTensorMode
    t = torch.zeros(8, 8, dtype=torch.float16)
    with pytest.raises(ValueError, match="device memory"):
        linear.gemm_linear(t, t, t)
    with pytest.raises(ValueError, match="device memory"):
        linear.gemm_linear_bwd(t, t, t, None, t, t)
    with FakeTensorMode():
        def e(*shape, dtype=torch.float16):
            return torch.empty(*shape, dtype=dtype, device="cuda")
        x, w, out = e(4, 16), e(16, 24), e(4, 24)
        for message, args, more in (
                ("x must be", (x, e(24, 16), out), {}), ("out must be", (x, w, e(4, 16)), {}), ("activation", (x, w, out), dict(activation="tanh")),
                ("columns of x", (e(16, 4).t(), w, out), {}), ("w must have contiguous", (x, e(32, 48)[::2, ::2], out), {}),
                ("bias", (x, w, out, e(23)), {}), ("bias", (x, w, out, e(24, dtype=torch.float64)), {}), ("residual must be", (x, w, out, None, x), {}),
                ("out must have the type", (x, w, e(4, 24, dtype=torch.bfloat16)), {}), ("pre must be", (x, w, out, None, None, x), {}),
                ("workspace must be", (x, w, e(4, 24)), dict(workspace=e(4, 4)[:, :2], stream=0))):
            with pytest.raises(ValueError, match=message):
                linear.gemm_linear(*args, **{"stream": 0, **more})
        with pytest.raises(TypeError, match="float16 or bfloat16"):
            linear.gemm_linear(e(4, 16, dtype=torch.float32), w, out, stream=0)
        for message, args in (("one of dx", (out, x, w)), ("dx needs w", (out, x, None, None, x)), ("dw needs x", (out, None, w, None, None, w)),
                              ("dx needs w", (out, x, w, None, x, None, None, "relu")), ("dbias", (out, x, w, None, None, None, e(24))),
                              ("dx must be", (out, x, w, None, e(5, 16)))):
            with pytest.raises(ValueError, match=message):
                linear.gemm_linear_bwd(*args, stream=0)
    n = binding.native()
    for call, count in ((n.gemm_linear, 9), (n.gemm_linear_bwd, 10)):
        for args in ((), (t,) * count, (None,) * count, (1,) * count):
            assert call(*args) == n.NOT_PLAIN


def test_products_in_python_refuse_memory_that_they_cannot_use():
    """A workspace in host memory or with gaps, or a layout that is none, never reaches the library."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        def e(*shape, dtype=torch.float16, device="cuda"):
            return torch.empty(*shape, dtype=dtype, device=device)
        a, b, c = e(4, 512), e(512, 16), e(4, 16)
        space = 2 * 4 * 16 * 4
        for bad in (e(space, dtype=torch.uint8, device="cpu"), e(space, 2, dtype=torch.uint8)[:, 0]):
            with pytest.raises(ValueError, match="workspace"):
                linear.linear_product(a, b, linear.ROWS, c, 0, 2, bad, stream=0)
        for layout in (-1, 3, 1.5):
            with pytest.raises(ValueError, match="layout"):
                linear.linear_product(a, b, layout, c, 0, stream=0)
