"""Refusals of the 4-bit cache, its attention and the norms with rotation, without a GPU: the C ABI on pointers that are never
dereferenced, the Python path on tensors without storage."""
import ctypes
import os
import re

import pytest
import torch

from paper_2403_16863_amd import kv4, rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("header,module", [("kv4", kv4), ("qk_rope", rope)])
def test_every_declared_symbol_is_exported_and_bound(header, module):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header + ".h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b((?:kv4|qk)_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(module.SYMBOLS)
    for n in names:
        assert hasattr(module.lib(), n) and hasattr(module, n)


def p(x):
    return ctypes.c_void_p(x)


def test_append_refuses_bad_arguments():
    L = kv4.lib()

    def call(k=0x10000, v=0x20000, cache=0x30000, slots=0x40000, cos=0x50000, sin=0x60000, pos=0x70000, rows=8, T=4, heads=2, d=64, pages=3,
             page=16, dt=0, ts=128, hs=64):
        return L.kv4_append(p(k), ts, hs, p(v), ts, hs, p(cache), p(slots), p(cos), p(sin), p(pos), rows, 0, T, heads, d, pages, page, dt, None)
    for bad in (dict(k=0), dict(v=0), dict(cache=0), dict(slots=0), dict(k=0x10008), dict(cache=0x30004), dict(sin=0), dict(pos=0), dict(rows=0),
                dict(T=-1), dict(heads=0), dict(pages=0), dict(page=0), dict(page=8), dict(page=24), dict(page=1 << 17), dict(dt=2), dict(ts=100),
                dict(cos=0x50004)):
        assert call(**bad) == kv4.KV4_EINVAL, bad
    for bad in (dict(d=32), dict(d=96), dict(d=256), dict(pages=1 << 28), dict(T=1 << 30)):
        assert call(**bad) == kv4.KV4_EUNSUPPORTED, bad
    assert call(T=0) == kv4.KV4_OK                                  # nothing to launch
    assert L.kv4_read(p(0x30000), p(0x40000), None, None, 4, 2, 64, 3, 16, 0, None) == kv4.KV4_EINVAL
    assert L.kv4_read(p(0x30000), p(0x40000), p(0x10002), None, 4, 2, 64, 3, 16, 0, None) == kv4.KV4_EINVAL
    assert L.kv4_read(p(0x30000), p(0x40000), p(0x10000), None, 0, 2, 64, 3, 16, 0, None) == kv4.KV4_OK


def test_attention_refuses_bad_arguments():
    L = kv4.lib()

    def call(q=0x100000, cache=0x200000, tables=0x300000, lens=0x400000, cu=0x500000, out=0x600000, lse=0x700000, T=4, B=2, H=4, heads=2, d=64,
             pages=3, page=16, width=5, max_q=3, scale=0.1, dt=0, ws=0):
        return L.kv4_attn(p(q), p(cache), p(tables), p(lens), p(cu), p(out), p(lse), T, B, H, heads, d, pages, page, width, max_q, 1, scale, dt,
                          p(ws), 0, None)
    for bad in (dict(q=0), dict(cache=0), dict(tables=0), dict(lens=0), dict(out=0), dict(lse=0), dict(q=0x100008), dict(out=0x100000),
                dict(out=0x100040), dict(lse=0x600000), dict(T=-1), dict(B=0), dict(H=0), dict(H=5), dict(heads=0), dict(pages=0), dict(page=24),
                dict(width=0), dict(max_q=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(dt=7), dict(ws=0x800008), dict(lens=0x400002),
                dict(cu=0, T=5), dict(cu=0, max_q=3)):
        assert call(**bad) == kv4.KV4_EINVAL, bad
    for bad in (dict(d=96), dict(width=1 << 28), dict(pages=1 << 28), dict(B=65536), dict(T=1 << 30), dict(max_q=1 << 30)):
        assert call(**bad) == kv4.KV4_EUNSUPPORTED, bad
    assert call(T=0) == kv4.KV4_OK
    assert L.kv4_attn_workspace(2, 2, 5, 2, 64, 16, 5, 1) == kv4.KV4_EINVAL
    assert L.kv4_attn_workspace(1, 1, 4, 2, 64, 16, 2, 1) == 0         # no sequence that long is cut
    assert L.kv4_attn_workspace(1, 1, 4, 2, 64, 16, 500, 1) > 0


def test_rope_refuses_bad_arguments():
    L = rope.lib()

    def h(data, ts=256):
        return rope.Heads(data, 4096, ts, 64)

    def call(q=h(0x10000), k=h(0x20000), qo=h(0x30000), ko=h(0x40000), qw=0x50000, cos=0x60000, sin=0x70000, pos=0x80000, rows=9, eps=1e-6, B=2,
             N=3, H=4, Hkv=2, d=64, dt=0):
        return L.qk_norm_rope(q, k, qo, ko, p(qw), None, 0, p(cos), p(sin), p(pos), rows, eps, 0, B, N, H, Hkv, d, dt, None)
    for bad in (dict(q=h(0)), dict(q=h(0), qo=h(0), k=h(0), ko=h(0)), dict(qo=h(0x30004)), dict(k=h(0x20000, 100)), dict(qw=0x50004), dict(cos=0), dict(pos=0),
                dict(rows=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(B=0), dict(N=0), dict(dt=3)):
        assert call(**bad) == rope.QK_EINVAL, bad
    for bad in (dict(d=96), dict(B=1 << 16, N=1 << 16)):
        assert call(**bad) == rope.QK_EUNSUPPORTED, bad

    def back(qw=0x50000, dqw=0x51000, ws=0x90000, room=1 << 30, q=h(0x10000)):
        return L.qk_norm_rope_bwd(h(0x30000), h(0x40000), q, h(0), h(0xa0000), h(0xb0000), p(qw), None, 0, p(dqw), None, p(0x60000), p(0x70000),
                                  p(0x80000), 9, 1e-6, 0, 2, 3, 4, 2, 64, 0, p(ws), room, None)
    for bad in (dict(dqw=0), dict(qw=0), dict(ws=0), dict(room=100), dict(q=h(0)), dict(ws=0x90008)):
        assert back(**bad) == rope.QK_EINVAL, bad
    assert L.qk_norm_rope_bwd_workspace(0, 1, 1, 1, 64) == rope.QK_EINVAL


def test_python_refusals_name_the_argument():
    from torch._subclasses.fake_tensor import FakeTensorMode
    t = torch.zeros(4, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="device memory"):
        kv4.kv4_append(t, t, torch.zeros(3, 2, 16, 68, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="device memory"):
        rope.qk_norm_rope(t[None], None, t[None], None, torch.zeros(9, 32), torch.zeros(9, 32), torch.zeros(1, 4, dtype=torch.int32))
    with FakeTensorMode():
        z = lambda *s, dtype=torch.float16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        i32 = torch.int32
        cache, k, slots = z(3, 2, 16, 68, dtype=torch.uint8), z(4, 2, 64), z(4, dtype=i32)
        cos = z(9, 32, dtype=torch.float32)
        for match, args in (("cache", (k, k, z(3, 2, 16, 66, dtype=torch.uint8), slots)), ("cache", (k, k, cache.transpose(0, 1), slots)),
                            ("cache", (k, k, cache.view(torch.int8), slots)), ("shape", (z(4, 3, 64), z(4, 3, 64), cache, slots)),
                            ("shape", (k, z(5, 2, 64), cache, slots)), ("dtype", (k, k.bfloat16(), cache, slots)),
                            ("channels", (z(4, 64, 2).transpose(1, 2), k, cache, slots)), ("slots", (k, k, cache, z(5, dtype=i32))),
                            ("slots", (k, k, cache, slots.long())), ("together", (k, k, cache, slots, cos)), ("together", (k, k, cache, slots, cos, cos)),
                            ("sin", (k, k, cache, slots, cos, z(8, 32, dtype=torch.float32), slots)), ("cos", (k, k, cache, slots, cos.half(), cos, slots))):
            with pytest.raises(ValueError, match=match):
                kv4.kv4_append(*args)
        with pytest.raises(TypeError):
            kv4.kv4_append(k.float(), k.float(), cache, slots)
        for match, args in (("one of", (cache, slots)), ("shape|contiguous", (cache, slots, z(4, 3, 64))), ("dtype", (cache, slots, k, k.bfloat16()))):
            with pytest.raises(ValueError, match=match):
                kv4.kv4_read(*args)
        q, tables, lens, lse, cu = z(4, 4, 64), z(2, 5, dtype=i32), z(2, dtype=i32), z(4, 4, dtype=torch.float32), z(3, dtype=i32)
        for match, args in (("shape", (z(4, 4, 128), cache, tables, lens, q, lse, True, 1.0)), ("dtype", (q, cache, tables, lens, q.bfloat16(), lse, True, 1.0)),
                            ("lse", (q, cache, tables, lens, q, lse.half(), True, 1.0)), ("tables", (q, cache, lens, lens, q, lse, True, 1.0)),
                            ("lens", (q, cache, tables, cu, q, lse, True, 1.0)), ("cu_q", (q, cache, tables, lens, q, lse, True, 1.0, lens)),
                            ("max_q", (q, cache, tables, lens, q, lse, True, 1.0, cu)), ("T / B", (q, cache, z(3, 5, dtype=i32), cu, q, lse, True, 1.0)),
                            ("T / B", (q, cache, tables, lens, q, lse, True, 1.0, None, 3))):
            with pytest.raises(ValueError, match=match):
                kv4.kv4_attn(*args)
        x, y, pos = z(2, 3, 4, 64), z(2, 3, 2, 64), z(2, 3, dtype=i32)
        w = z(64)
        for match, args in (("together", (x, y, x, None, cos, cos, pos)), ("together", (None, None, None, None, cos, cos, pos)), ("heads", (x, y, y, y, cos, cos, pos)),
                            ("sizes", (x, z(2, 4, 2, 64), x, z(2, 4, 2, 64), cos, cos, pos)), ("dtype", (x, y.bfloat16(), x, y, cos, cos, pos)),
                            ("channels", (z(2, 3, 64, 4).transpose(2, 3), y, x, y, cos, cos, pos)), ("positions", (x, y, x, y, cos, cos, pos.long())),
                            ("sin", (x, y, x, y, cos, z(9, 64, dtype=torch.float32), pos)), ("weights", (x, y, x, y, cos, cos, pos, w, w.float())),
                            ("weights", (x, y, x, y, cos, cos, pos, z(32)))):
            with pytest.raises(ValueError, match=match):
                rope.qk_norm_rope(*args)
        with pytest.raises(TypeError):
            rope.qk_norm_rope(x.float(), None, x.float(), None, cos, cos, pos)
        with pytest.raises(ValueError, match="gradient go together"):
            rope.qk_norm_rope_bwd(x, None, x, None, x, None, cos, cos, pos, w)
        with pytest.raises(ValueError, match="forward's input"):
            rope.qk_norm_rope_bwd(x, None, None, None, x, None, cos, cos, pos, w, None, w.float())


def test_sizes_at_the_limits_of_32_bits():
    """No launch of 2^32 threads (16 waves to each of 2^22 rows of q), no tile whose end passes 2^31 keys, no sequences at all."""
    L = kv4.lib()
    assert L.kv4_attn_workspace(1 << 17, 1, 32, 8, 64, 16, 500, 1) == 0
    assert L.kv4_attn_workspace((1 << 17) - 1, 1, 32, 8, 64, 16, 500, 1) > 0
    many = 1 << 14                                                       # segments enough to stay whole
    assert L.kv4_attn_workspace(many, many, 8, 8, 64, 65536, 32767, 1) == 0
    assert L.kv4_attn_workspace(many, many, 8, 8, 64, 16, (1 << 27) - 4096, 1) == 0
    assert L.kv4_attn_workspace(many, many, 8, 8, 64, 16, (1 << 27) - 4095, 1) == kv4.KV4_EUNSUPPORTED
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        z = lambda *s, dtype=torch.float16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        i32, f32 = torch.int32, torch.float32
        cache, q = z(3, 2, 16, 68, dtype=torch.uint8), z(0, 4, 64)
        kv4.kv4_attn(q, cache, z(0, 5, dtype=i32), z(0, dtype=i32), q, z(0, 4, dtype=f32), True, 1.0)
        kv4.kv4_attn(q, cache, z(2, 5, dtype=i32), z(2, dtype=i32), q, z(0, 4, dtype=f32), True, 1.0)


def test_attention_refuses_caches_of_too_many_groups():
    L = kv4.lib()

    def call(pages, heads, cache=0x200000):
        return L.kv4_attn(p(0x100000), p(cache), p(0x300000), p(0x400000), p(0x500000), p(0x600000), p(0x700000), 4, 2, heads, heads, 64, pages, 16,
                          5, 3, 1, 0.1, 0, None, 0, None)
    assert call(1 << 26, 64) == kv4.KV4_EUNSUPPORTED               # 2^32 groups of 16 tokens
    assert call((1 << 27) - 1, 32) == kv4.KV4_EINVAL               # fewer, but out within them
