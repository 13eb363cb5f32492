"""Outputs of the norms that begin where another tensor does, without a GPU."""
import ctypes

from paper_2403_16863_amd import rope


def p(x):
    return ctypes.c_void_p(x)


def h(data, batch=4096, token=256, head=64):
    return rope.Heads(data, batch, token, head)


def forward(q=h(0x10000), k=h(0x20000), qo=h(0x30000), ko=h(0x40000), B=2, N=3, H=4, Hkv=2):
    return rope.lib().qk_norm_rope(q, k, qo, ko, None, None, 0, p(0x60000), p(0x70000), p(0x80000), 9, 1e-6, 0, B, N, H, Hkv, 64, 0, None)


def backward(dqo=h(0x10000), dko=h(0x20000), q=h(0x30000), k=h(0x40000), dq=h(0x50000), dk=h(0x58000)):
    return rope.lib().qk_norm_rope_bwd(dqo, dko, q, k, dq, dk, p(0x90000), p(0x91000), 0, p(0x92000), p(0x93000), p(0x60000), p(0x70000), p(0x80000), 9,
                                       1e-6, 0, 2, 3, 4, 2, 64, 0, p(0xa0000), 1 << 30, None)


def test_forward_refuses_outputs_over_other_memory():
    for bad in (dict(qo=h(0x10000, token=64, head=192)), dict(qo=h(0x10000, batch=2048)), dict(qo=h(0x20000)), dict(ko=h(0x10000)), dict(ko=h(0x30000))):
        assert forward(**bad) == rope.QK_EINVAL, bad


def test_backward_refuses_outputs_over_other_memory():
    for bad in (dict(dq=h(0x10000, head=128)), dict(dq=h(0x20000)), dict(dk=h(0x10000)), dict(dk=h(0x50000)), dict(dq=h(0x30000, head=128)),
                dict(dq=h(0x40000))):
        assert backward(**bad) == rope.QK_EINVAL, bad


def test_in_place_is_not_refused_for_it():
    """Nothing can be launched here, so a call that passes the checks is refused by the runtime, or succeeds where there is a device's."""
    import torch
    if torch.cuda.is_available():
        return                                                     # the addresses are nobody's
    assert forward(qo=h(0x10000)) == rope.QK_ELAUNCH
    assert forward(qo=h(0x10000, batch=0, token=8), B=1, N=1) == rope.QK_ELAUNCH       # strides of a size of 1 are not looked at
    assert forward(k=h(0x30000), ko=h(0x30000), Hkv=0) == rope.QK_ELAUNCH              # nor is a tensor of no heads
    assert backward(dq=h(0x10000), dk=h(0x20000)) == rope.QK_ELAUNCH
