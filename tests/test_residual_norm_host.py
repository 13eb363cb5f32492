"""Refusals of the norms with the residual stream without a GPU: the C ABI on pointers that are never dereferenced, the Python path on
tensors of the CPU or without storage."""
import ctypes
import os
import re

import pytest
import torch

from paper_2403_16863_amd import binding, norm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ON_CPU = not torch.cuda.is_available()


def p(x):
    return ctypes.c_void_p(x)


def t(data, batch=192, token=64):
    return norm.Tokens(data, batch, token)


NONE = t(None)


def vec(gate=0x90000, stride=64, gate_f32=0, post=0xa0000, pre=0xb0000, f32=1, alpha=1.0, eps=1e-6):
    return norm.Vectors(gate, stride, gate_f32, post, pre, f32, alpha, eps)


# 2 sequences of 3 tokens of 64 channels: 768 bytes
def forward(x=t(0x10000), h=t(0x20000), y=t(0x30000), z=t(0x40000), v=vec(), B=2, N=3, C=64, dt=0):
    return norm.lib().residual_norm(x, h, y, z, v, B, N, C, dt, None)


def backward(dy=t(0x10000), dz=t(0x20000), y=t(0x30000), h=t(0x40000), dx=t(0x50000), dh=t(0x60000), v=vec(), dg=0xc0000, dpo=0xd0000, dpr=0xe0000, B=2,
             N=3, C=64, dt=1, ws=0x100000, bytes_=1 << 20):
    return norm.lib().residual_norm_bwd(dy, dz, y, h, dx, dh, v, p(dg), p(dpo), p(dpr), B, N, C, dt, p(ws), bytes_, None)


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "residual_norm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b((?:residual_norm|norm_strerror)[a-z_0-9]*)\s*\(", text)))
    assert names == sorted(norm.SYMBOLS)
    for n in names:
        assert hasattr(norm.lib(), n) and hasattr(norm, n)


def test_forward_refuses_bad_arguments():
    bad_values = [dict(x=NONE), dict(y=NONE, z=NONE), dict(z=NONE), dict(v=vec(pre=None)), dict(h=NONE), dict(h=NONE, y=NONE),
                  dict(h=NONE, y=NONE, v=vec(gate=None, post=None, alpha=0.5)), dict(x=t(0x10008)), dict(y=t(0x30002)), dict(B=0), dict(N=0), dict(N=-1),
                  dict(C=0), dict(dt=2), dict(dt=-1), dict(v=vec(alpha=float("nan"))), dict(v=vec(alpha=float("inf"))), dict(v=vec(eps=-1e-6)),
                  dict(v=vec(eps=float("nan"))), dict(v=vec(gate=0x90004)), dict(v=vec(stride=56)), dict(v=vec(stride=68)), dict(v=vec(stride=-64)),
                  dict(v=vec(post=0xa0008)), dict(v=vec(pre=0xb0001)), dict(x=t(0x10000, 192, 60)), dict(x=t(0x10000, 190)), dict(x=t(0x10000, -192)),
                  dict(y=t(0x30000, 192, 56)), dict(y=t(0x30000, 128)), dict(y=t(0x30000, 0)), dict(z=t(0x40000, 64, 64)), dict(x=t(0x10000, 1 << 60))]
    for bad in bad_values:
        assert forward(**bad) == norm.NORM_EINVAL, bad
    for bad in (dict(C=60), dict(C=16392), dict(B=1 << 20, N=1 << 12)):
        assert forward(**bad) == norm.NORM_EUNSUPPORTED, bad


def test_outputs_over_other_memory_are_refused():
    for bad in (dict(y=t(0x10000 + 16)), dict(y=t(0x10000, 256)), dict(z=t(0x20000 + 752)), dict(y=t(0x40000)), dict(z=t(0x30000 + 128)), dict(y=t(0x90000)),
                dict(z=t(0xa0000 - 752)), dict(z=t(0xb0000)), dict(x=t(0x10000, 384, 128), y=t(0x10000 + 112, 384, 128))):
        assert forward(**bad) == norm.NORM_EINVAL, bad
    for bad in (dict(dx=t(0x10000 + 128)), dict(dx=t(0x20000, 256)), dict(dh=t(0x50000)), dict(dh=t(0x40000 + 16)), dict(dx=t(0x90000)), dict(dh=t(0xc0000)),
                dict(dx=t(0xd0000)), dict(dh=t(0x100000)), dict(dg=0xd0000), dict(dpo=0xe0000 + 16), dict(dpr=0x10000), dict(dg=0x90000), dict(dpo=0xa0000),
                dict(ws=0x50000 - 256), dict(ws=0xb0000)):
        assert backward(**bad) == norm.NORM_EINVAL, bad


def test_backward_refuses_bad_arguments():
    for bad in (dict(dy=NONE, dz=NONE), dict(dz=NONE), dict(v=vec(pre=None)), dict(y=NONE), dict(h=NONE), dict(dx=NONE, dh=NONE), dict(v=vec(gate=None)),
                dict(v=vec(post=None)), dict(dg=0xc0004), dict(dpo=0xd0008), dict(dpr=0xe0001), dict(ws=0), dict(ws=0x100008), dict(bytes_=64), dict(B=0), dict(C=0),
                dict(dt=5), dict(dx=t(0x50000, 0)), dict(dh=t(0x60000, 192, 0)), dict(dy=t(0x10000, 190)), dict(v=vec(eps=float("inf")))):
        assert backward(**bad) == norm.NORM_EINVAL, bad
    for bad in (dict(C=60), dict(C=16392), dict(B=1 << 20, N=1 << 12)):
        assert backward(**bad) == norm.NORM_EUNSUPPORTED, bad


@pytest.mark.skipif(not ON_CPU, reason="the addresses are nobody's")
def test_what_is_not_refused():
    """Nothing can be launched here, so a call that passes the checks is refused by the runtime."""
    for good in (dict(), dict(y=NONE), dict(z=NONE, v=vec(pre=None)), dict(h=NONE, y=NONE, v=vec(gate=None, post=None)), dict(y=t(0x10000)), dict(y=t(0x20000)),
                 dict(y=t(0x10000), z=t(0x20000)), dict(x=t(0x10000, 0, 0)), dict(y=t(0x30000, 64, 128)), dict(B=1, y=t(0x30000, -5)),
                 dict(x=t(0x10000, 384, 128), y=t(0x10000 + 128, 384, 128)), dict(v=vec(stride=0))):
        assert forward(**good) == norm.NORM_ELAUNCH, good
    for good in (dict(), dict(dy=NONE), dict(dz=NONE, y=NONE, dpr=0, v=vec(pre=None)), dict(dx=NONE), dict(dh=NONE), dict(dg=0, dpo=0, dpr=0, ws=0, bytes_=0),
                 dict(dx=t(0x10000)), dict(dx=t(0x40000), dh=t(0x20000)), dict(h=NONE, dg=0, dpo=0, v=vec(gate=None, post=None)), dict(v=vec(stride=0))):
        assert backward(**good) == norm.NORM_ELAUNCH, good


def test_workspaces_by_size():
    assert norm.residual_norm_bwd_workspace(1, 1, 64) == 4 * 64 * 2
    assert norm.residual_norm_bwd_workspace(2, 4096, 4096, True) > norm.residual_norm_bwd_workspace(2, 4096, 4096)
    for bad in ((0, 1, 8), (1, 1, 12), (1, 2 ** 31, 8), (1 << 16, 1 << 16, 8)):
        with pytest.raises(norm.NormError):
            norm.residual_norm_bwd_workspace(*bad)


def test_python_names_what_it_refuses():
    from torch._subclasses.fake_tensor import FakeTensorMode
    c = torch.zeros(1, 2, 8, dtype=torch.float16)
    w = torch.ones(8)
    with pytest.raises(ValueError, match="device"):
        norm.residual_norm(c, None, None, c.clone(), None, None, w)
    with pytest.raises(ValueError, match="device"):
        norm.residual_norm_bwd(c, None, None, None, c.clone(), None)
    with FakeTensorMode():
        def e(*shape, dtype=torch.float16):
            return torch.empty(*shape, dtype=dtype, device="cuda")
        x, v = e(2, 3, 16), e(16)
        for message, args, more in (
                ("one of y and z", (x, x, None, None), {}), ("go together", (x, x, e(2, 3, 16), x), {}), ("without h", (x, None, x, None), {}),
                ("without h", (x, None, None, x, v, None, v), {}), ("without h", (x, None, None, x, None, None, v), dict(alpha=2.0)),
                ("gate must be", (x, x, x, None, e(3, 16)), {}), ("gate must be", (x, x, x, None, e(16, dtype=torch.float64)), {}),
                ("rows of gate", (x, x, x, None, e(16).expand(2, 16)), {}), ("post_weight", (x, x, x, None, None, e(8)), {}),
                ("one type", (x, x, x, x, None, v, e(16, dtype=torch.float32)), {}), ("h must be", (x, e(2, 3, 8), x, None), {}),
                ("channels of y", (x, x, e(2, 16, 3).transpose(1, 2), None), {}), ("y must have the type", (x, x, e(2, 3, 16, dtype=torch.bfloat16), None), {})):
            with pytest.raises(ValueError, match=message):
                norm.residual_norm(*args, **{"stream": 0, **more})
        with pytest.raises(TypeError, match="float16 or bfloat16"):
            norm.residual_norm(e(2, 3, 16, dtype=torch.float32), x, x, None, stream=0)
        for message, args in (("one of dy", (None, None, x, x, x, x)), ("one of dy", (x, None, x, x, None, None)), ("dz goes", (x, x, x, x, x, x)),
                              ("dz goes", (x, x, None, x, x, x, None, None, v)), ("needs the forward's h", (x, None, None, None, x, x, v)),
                              ("dgate has no", (x, None, None, None, x, x, None, None, None, v)),
                              ("dgate must be", (x, None, None, x, x, x, v, None, None, e(16)))):
            with pytest.raises(ValueError, match=message):
                norm.residual_norm_bwd(*args, stream=0)
    n = binding.native()
    for call, count in ((n.residual_norm, 10), (n.residual_norm_bwd, 16)):
        for args in ((), (c,) * count, (None,) * count, (1,) * count):
            assert call(*args) == n.NOT_PLAIN
