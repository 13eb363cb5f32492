"""Refusals of the rotation by several axes without a GPU, and the axes of pairs."""
import ctypes

import pytest
import torch

from paper_2403_16863_amd import binding, rope


def p(x):
    return ctypes.c_void_p(x)


def h(data, batch=4096, token=256, head=64):
    return rope.Heads(data, batch, token, head)


GOOD = rope.axes_of_pairs((8, 12, 12), 64)


def forward(axes=3, of_pair=GOOD, qo=h(0x30000), d=64, positions=0x80000):
    return rope.lib().qk_norm_rope_axes(h(0x10000), h(0x20000), qo, h(0x40000), None, None, 0, p(0x60000), p(0x70000), p(positions), 9, axes, of_pair, 1e-6, 0,
                                        2, 3, 4, 2, d, 0, None)


def backward(axes=3, of_pair=GOOD, dq=h(0x50000), d=64, ws=0xa0000):
    return rope.lib().qk_norm_rope_axes_bwd(h(0x10000), h(0x20000), h(0x30000), h(0x40000), dq, h(0x58000), p(0x90000), p(0x91000), 0, p(0x92000), p(0x93000),
                                            p(0x60000), p(0x70000), p(0x80000), 9, axes, of_pair, 1e-6, 0, 2, 3, 4, 2, d, 0, p(ws), 1 << 30, None)


def test_refusals():
    for call in (forward, backward):
        for bad in (dict(axes=0), dict(axes=-1), dict(axes=5), dict(axes=2), dict(of_pair=None), dict(of_pair=b"\0" * 31 + b"\3"), dict(of_pair=b"\0" * 31 + b"\x0f"),
                    dict(of_pair=b"\0" * 31 + b"\xfe")):
            assert call(**bad) == rope.QK_EINVAL, bad
        assert call(d=96, of_pair=b"\0" * 48) == rope.QK_EUNSUPPORTED
    assert forward(qo=h(0x20000)) == rope.QK_EINVAL and forward(positions=0) == rope.QK_EINVAL
    assert backward(dq=h(0x20000)) == rope.QK_EINVAL and backward(ws=0) == rope.QK_EINVAL
    if not torch.cuda.is_available():                                  # the addresses are nobody's
        for call in (forward, backward):
            for good in (dict(), dict(of_pair=b"\xff" * 32), dict(axes=4, of_pair=bytes(i % 4 for i in range(32)))):
                assert call(**good) == rope.QK_ELAUNCH


def test_gradients_of_weights_over_other_memory_are_refused():
    """One tensor for both weights' gradients, or the sums' own memory, in both forms of the call."""
    def call(by_axes, dqw=0x92000, dkw=0x93000, qw=0x90000, kw=0x91000, f32=0, ws=0xa0000):
        L, more = rope.lib(), (3, GOOD) if by_axes else ()
        return (L.qk_norm_rope_axes_bwd if by_axes else L.qk_norm_rope_bwd)(
            h(0x10000), h(0x20000), h(0x30000), h(0x40000), h(0x50000), h(0x58000), p(qw), p(kw), f32, p(dqw), p(dkw), p(0x60000), p(0x70000), p(0x80000), 9, *more,
            1e-6, 0, 2, 3, 4, 2, 64, 0, p(ws), 1 << 30, None)
    for by_axes in (False, True):
        for bad in (dict(dkw=0x92000), dict(dkw=0x92000 + 252), dict(dqw=0x93000 + 4), dict(ws=0x92000), dict(ws=0x93000 - 16), dict(ws=0x90000), dict(ws=0x91000 + 112),
                    dict(ws=0x91000 + 240, f32=1)):
            assert call(by_axes, **bad) == rope.QK_EINVAL, bad
        if not torch.cuda.is_available():
            for good in (dict(), dict(dkw=0x92000 + 256), dict(ws=0x91000 + 128), dict(ws=0x91000 + 256, f32=1)):
                assert call(by_axes, **good) == rope.QK_ELAUNCH, good


def test_axes_of_pairs():
    assert rope.axes_of_pairs((1, 2, 3), 16) == bytes([0, 1, 1, 2, 2, 2, 255, 255])
    assert rope.axes_of_pairs((1, 2, 3), 16, alternating=True) == bytes([0, 1, 2, 1, 2, 2, 255, 255])
    assert rope.axes_of_pairs((32,), 64) == bytes(32) and rope.axes_of_pairs((0, 0), 64) == b"\xff" * 32
    for bad in ((), (1, 2, 3, 4, 5), (33,), (-1, 2), (20, 13)):
        with pytest.raises(ValueError, match="sections"):
            rope.axes_of_pairs(bad, 64)


def test_python_names_what_it_refuses():
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        def e(*shape, dtype=torch.float16):
            return torch.empty(*shape, dtype=dtype, device="cuda")
        q, t, at = e(2, 3, 4, 64), e(9, 32, dtype=torch.float32), e(2, 3, 3, dtype=torch.int32)
        for message, positions, axes in (("positions must be", e(2, 3, dtype=torch.int32), GOOD), ("positions must be", e(2, 3, 3, dtype=torch.int64), GOOD),
                                         ("positions must be", e(3, 2, 3, dtype=torch.int32).transpose(0, 1), GOOD), ("bytes", at, list(GOOD)), ("bytes", at, GOOD[:31]),
                                         ("bytes", at, GOOD * 2), ("axes name", at, b"\3" * 32), ("1 to 4", e(2, 3, 5, dtype=torch.int32), GOOD)):
            with pytest.raises(ValueError, match=message):
                rope.qk_norm_rope_axes(q, None, e(2, 3, 4, 64), None, t, t, positions, axes, stream=0)
            with pytest.raises(ValueError, match=message):
                rope.qk_norm_rope_axes_bwd(q, None, None, None, e(2, 3, 4, 64), None, t, t, positions, axes, stream=0)
    n = binding.native()
    for call, count in ((n.qk_norm_rope_axes, 13), (n.qk_norm_rope_axes_bwd, 18)):
        for args in ((), (None,) * count, (1,) * count, (torch.zeros(1, 1, 1, 64),) * count):
            assert call(*args) == n.NOT_PLAIN
