"""Sizes of the cache's calls whose products pass 64 bits: refused, without a GPU."""
import ctypes

from paper_2403_16863_amd import kv4


def p(x):
    return ctypes.c_void_p(x)


def test_segments_that_wrap_around_are_refused():
    """2^15 sequences of 2^30 rows in each of 2^26 heads are 2^64 row blocks and more."""
    L, heads = kv4.lib(), 1 << 26
    for width in (2, 1000):
        assert L.kv4_attn_workspace(1, 1 << 15, heads, heads, 64, 16, width, 1 << 30) == kv4.KV4_EUNSUPPORTED
        assert L.kv4_attn(p(0x100000), p(1 << 44), p(0x300000), p(0x400000), p(0x500000), p(1 << 45), p(0x700000), 1, 1 << 15, heads, heads, 64, 1, 16,
                          width, 1 << 30, 1, 0.1, 0, None, 0, None) == kv4.KV4_EUNSUPPORTED
    assert L.kv4_attn_workspace(1, 65535, (1 << 31) - 1, (1 << 31) - 1, 64, 16, 2, 1 << 30) == kv4.KV4_EUNSUPPORTED


def test_threads_that_wrap_around_are_refused():
    L, T, heads = kv4.lib(), (1 << 31) - 1, 1 << 30
    assert L.kv4_append(p(0x10000), 64, 64, p(0x20000), 64, 64, p(0x30000), p(0x40000), None, None, None, 0, 0, T, heads, 128, 3, 16, 0,
                        None) == kv4.KV4_EUNSUPPORTED
    assert L.kv4_read(p(0x30000), p(0x40000), p(0x10000), None, T, heads, 128, 3, 16, 0, None) == kv4.KV4_EUNSUPPORTED


def test_python_sizes_beyond_an_int_are_refused():
    """Not cut to 32 bits: 2^32 + 1 queries of a sequence are not one."""
    import pytest
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode

    from paper_2403_16863_amd import rope
    for bad in ((1, 1, 4, 2, 64, 16, 500, (1 << 32) + 1), (1, 1, 4, 2, 64, 16, (1 << 32) + 500, 1), (1 << 40, 1, 4, 2, 64, 16, 500, 1)):
        with pytest.raises(kv4.Kv4Error) as e:
            kv4.kv4_attn_workspace(*bad)
        assert e.value.code == kv4.KV4_EUNSUPPORTED
    with pytest.raises(rope.RopeError) as e:
        rope.qk_norm_rope_bwd_workspace(1, (1 << 32) + 1, 4, 2, 64)
    assert e.value.code == rope.QK_EUNSUPPORTED
    with FakeTensorMode():
        z = lambda *s, dtype=torch.float16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        i32, many = torch.int32, (1 << 32) + 4
        cache, q, lens, cu = z(3, 2, 16, 68, dtype=torch.uint8), z(4, 4, 64), z(2, dtype=i32), z(3, dtype=i32)
        k = z(1, 2, 64).expand(many, 2, 64)
        for call in (lambda: kv4.kv4_attn(q, cache, z(2, 5, dtype=i32), lens, q, z(4, 4, dtype=torch.float32), True, 1.0, cu, (1 << 32) + 1),
                     lambda: kv4.kv4_append(k, k, cache, z(many, dtype=i32)),
                     lambda: kv4.kv4_read(cache, z(many, dtype=i32), z(many, 2, 64))):
            with pytest.raises(kv4.Kv4Error) as e:
                call()
            assert e.value.code == kv4.KV4_EUNSUPPORTED


def test_attention_refuses_outputs_and_scratch_memory_over_its_inputs():
    L = kv4.lib()
    q, cache, out, lse, ws, cap = 0x1000000, 0x2000000, 0x3000000, 0x4000000, 0x5000000, 64
    need = L.kv4_attn_workspace(4, 2, 4, 2, 64, 16, 500, 3)
    assert need > 0

    def call(q=q, cache=cache, out=out, lse=lse, ws=ws, room=need):
        return L.kv4_attn(p(q), p(cache), p(0x6000000), p(0x7000000), p(0x8000000), p(out), p(lse), 4, 2, 4, 2, cap, 3, 16, 500, 3, 1, 0.1, 0, p(ws),
                          room, None)
    # T * H * d * 2 = 2048 bytes of q and out, 64 of lse, 3 * 2 * 16 * 68 = 6528 of the cache
    for bad in (dict(lse=q), dict(lse=q + 2044), dict(lse=cache + 6524), dict(lse=cache - 60), dict(ws=q), dict(ws=q - need + 16), dict(ws=out + 2032),
                dict(ws=lse + 48), dict(ws=cache + 6512), dict(ws=cache - need + 16)):
        assert call(**bad) == kv4.KV4_EINVAL, bad


def test_reads_refuse_outputs_over_each_other_or_the_cache():
    L = kv4.lib()
    # 4 * 2 * 64 * 2 = 1024 bytes of k and v, 3 * 2 * 16 * 68 = 6528 of the cache

    def call(k=0x10000, v=0x20000, cache=0x30000):
        return L.kv4_read(p(cache), p(0x40000), p(k), p(v), 4, 2, 64, 3, 16, 0, None)
    for bad in (dict(k=0x20000), dict(k=0x20000 + 1008), dict(v=0x10000 - 1008), dict(k=0x30000), dict(v=0x30000 + 6512), dict(k=0x30000 - 1008)):
        assert call(**bad) == kv4.KV4_EINVAL, bad
