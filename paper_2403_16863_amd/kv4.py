"""Thin ctypes binding over the C ABI declared in include/kv4.h: a paged cache of keys and values in 4 bits, and the
attention over it.

    cache = torch.zeros(kv4.kv4_cache_shape(pages, heads, page_size, d), dtype=torch.uint8, device="cuda")
    kv4.kv4_append(k, v, cache, slots, cos, sin, positions)          # rotates the keys on the way
    kv4.kv4_attn(q, cache, tables, lens, out, lse, causal=True, scale=d ** -0.5)

Argument marshalling only: every step runs in the HIP kernels of libattn.so.  There is no fallback: if the library
has not been built, loading it fails loudly.
"""
from __future__ import annotations

import ctypes

from . import binding

KV4_F16, KV4_BF16 = 0, 1
KV4_OK, KV4_EINVAL, KV4_EUNSUPPORTED, KV4_ELAUNCH = 0, -1, -2, -3

# every symbol include/kv4.h declares
SYMBOLS = ("kv4_append", "kv4_read", "kv4_attn", "kv4_attn_workspace", "kv4_strerror")

_ready = False


def lib():
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i, f, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_longlong
        L.kv4_append.restype = i
        L.kv4_append.argtypes = [vp, ll, ll, vp, ll, ll, vp, vp, vp, vp, vp] + [i] * 8 + [vp]
        L.kv4_read.restype = i
        L.kv4_read.argtypes = [vp] * 4 + [i] * 6 + [vp]
        L.kv4_attn.restype = i
        L.kv4_attn.argtypes = [vp] * 7 + [i] * 10 + [f, i, vp, ll, vp]
        L.kv4_attn_workspace.restype = ll
        L.kv4_attn_workspace.argtypes = [i] * 8
        L.kv4_strerror.restype = ctypes.c_char_p
        L.kv4_strerror.argtypes = [i]
        _ready = True
    return L


def kv4_strerror(code: int) -> str:
    return lib().kv4_strerror(int(code)).decode()


class Kv4Error(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {kv4_strerror(code)} (code {code})")
        self.code = code


def kv4_cache_shape(pages: int, heads: int, page_size: int, d: int):
    """The shape of a cache, a contiguous uint8 tensor: page_size a power of two from 16, d 64 or 128."""
    return int(pages), int(heads), int(page_size), int(d) + int(d) // 16


def _cache(cache):
    """(pages, heads, page_size, d) of a cache."""
    import torch
    if cache.dtype != torch.uint8 or cache.dim() != 4 or not cache.is_contiguous() or cache.shape[3] % 17:
        raise ValueError("cache must be contiguous uint8 [pages,heads,page_size,d + d/16]")
    return cache.shape[0], cache.shape[1], cache.shape[2], cache.shape[3] // 17 * 16


def _devices(like, given):
    for name, t in given:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must live in device memory")
        if t.device != like.device:
            raise ValueError(f"{name} must live on the device of the other tensors")


def _ints(name, t, shape):
    import torch
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 {list(shape)}")


def _fit(what, *sizes):
    """The library counts in 32 bits, and ctypes would cut a larger number to them."""
    if max(sizes) > 2 ** 31 - 1 or min(sizes) < -2 ** 31:
        raise Kv4Error(KV4_EUNSUPPORTED, what)


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float16:
        return KV4_F16
    if t.dtype == torch.bfloat16:
        return KV4_BF16
    raise TypeError(f"queries, keys and values must be float16 or bfloat16, got {t.dtype}")


def _stream(stream, device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _first(name):
    """The native module's function of that name, from the first call on (one lookup a call)."""
    def first(*args):
        lib()
        globals()["_plain_" + name] = call = getattr(binding.native(), "kv4_" + name)
        return call(*args)
    return first


_plain_append, _plain_read, _plain_attn = _first("append"), _first("read"), _first("attn")


def kv4_append(k, v, cache, slots, cos=None, sin=None, positions=None, interleaved: bool = False, stream=None) -> None:
    """Slot slots[t] of the cache <- k[t], rotated by positions[t], and v[t], for k and v [T,heads,d] (any strides that divide by
    8, channels contiguous).  Tokens whose slot lies outside the cache (-1: padding) are left out; the others' slots must
    differ.  cos, sin: float32 [rows,d/2], or None for keys that need no rotation (any more).  Asynchronous on `stream` (an
    integer hipStream_t; default: torch's current stream)."""
    rc = _plain_append(k, v, cache, slots, cos, sin, positions, interleaved, stream)
    if not rc:
        return
    if rc < 0:
        raise Kv4Error(rc, "kv4_append")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    _devices(cache, (("cache", cache), ("k", k), ("v", v), ("slots", slots), ("cos", cos), ("sin", sin), ("positions", positions)))
    pages, heads, page_size, d = _cache(cache)
    if k.dim() != 3 or v.shape != k.shape or tuple(k.shape[1:]) != (heads, d):
        raise ValueError(f"k and v must share one [T,{heads},{d}] shape")
    if v.dtype != k.dtype:
        raise ValueError("k and v must share one dtype")
    if k.stride(2) != 1 or v.stride(2) != 1:
        raise ValueError("the channels of k and v must be contiguous")
    T, dt, rows = k.shape[0], _dtype_code(k), 0
    _ints("slots", slots, (T,))
    if (cos is None) != (sin is None) or (cos is not None and positions is None):
        raise ValueError("cos, sin and positions go together")
    if cos is not None:
        for name, t in (("cos", cos), ("sin", sin)):
            if t.dtype != torch.float32 or t.dim() != 2 or t.shape[1] != d // 2 or t.shape != cos.shape or not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous float32 [rows,d/2]")
        _ints("positions", positions, (T,))
        rows = cos.shape[0]
    _fit("kv4_append", T, rows, pages)
    ks, vs = ([t.stride(0) if T > 1 else 0, t.stride(1) if heads > 1 else 0] for t in (k, v))
    if T == 0:
        return
    with torch.cuda.device(cache.device):
        rc = lib().kv4_append(k.data_ptr(), *ks, v.data_ptr(), *vs, cache.data_ptr(), slots.data_ptr(), _ptr(cos), _ptr(sin), _ptr(positions),
                              rows, int(bool(interleaved)), T, heads, d, pages, page_size, dt, _stream(stream, cache.device))
    if rc != KV4_OK:
        raise Kv4Error(rc, "kv4_append")


def kv4_read(cache, slots, k=None, v=None, stream=None) -> None:
    """k, v [T,heads,d] (contiguous; either may be None) <- what slot slots[t] of the cache holds, zeros for a slot outside it."""
    rc = _plain_read(cache, slots, k, v, stream)
    if not rc:
        return
    if rc < 0:
        raise Kv4Error(rc, "kv4_read")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    like = k if k is not None else v
    if like is None:
        raise ValueError("one of k and v must be there")
    _devices(cache, (("cache", cache), ("slots", slots), ("k", k), ("v", v)))
    pages, heads, page_size, d = _cache(cache)
    for name, t in (("k", k), ("v", v)):
        if t is not None and (t.dim() != 3 or t.shape != like.shape or tuple(t.shape[1:]) != (heads, d) or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous [T,{heads},{d}]")
        if t is not None and t.dtype != like.dtype:
            raise ValueError("k and v must share one dtype")
    T, dt = like.shape[0], _dtype_code(like)
    _ints("slots", slots, (T,))
    _fit("kv4_read", T, pages)
    if T == 0:
        return
    with torch.cuda.device(cache.device):
        rc = lib().kv4_read(cache.data_ptr(), slots.data_ptr(), _ptr(k), _ptr(v), T, heads, d, pages, page_size, dt,
                            _stream(stream, cache.device))
    if rc != KV4_OK:
        raise Kv4Error(rc, "kv4_read")


def kv4_attn_workspace(T: int, B: int, H: int, heads: int, d: int, page_size: int, width: int, max_q: int) -> int:
    """Bytes of scratch memory that kv4_attn has a use for (0: none)."""
    sizes = [int(x) for x in (T, B, H, heads, d, page_size, width, max_q)]
    _fit("kv4_attn_workspace", *sizes)
    n = lib().kv4_attn_workspace(*sizes)
    if n < 0:
        raise Kv4Error(n, "kv4_attn_workspace")
    return n


def kv4_attn(q, cache, tables, lens, out, lse, causal: bool, scale: float, cu_q=None, max_q=None, workspace=None, stream=None) -> None:
    """out [T,H,d], lse [T,H] <- attention of q [T,H,d] over the cache.  Sequence b has lens[b] keys in the pages tables[b] and, with cu_q
    (int32 [B+1]), the queries cu_q[b] .. cu_q[b+1] - 1, at most max_q of them; without it T / B queries.  causal: the
    last query of a sequence sees its last key.  Nothing is recorded for autograd.  All contiguous; tables int32 [B,width], lens int32 [B], lse float32.

    Few long sequences are cut into runs of keys for which the call needs scratch memory: `workspace` (uint8,
    kv4_attn_workspace bytes), or, on torch's current stream, memory that it takes from torch's allocator itself (the graph's own
    pool while torch records one).  On another stream, or in a recording begun elsewhere, the keys are not cut without a workspace, which
    is slower."""
    rc = _plain_attn(q, cache, tables, lens, out, lse, causal, scale, cu_q, max_q, workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise Kv4Error(rc, "kv4_attn")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    _devices(cache, (("cache", cache), ("q", q), ("tables", tables), ("lens", lens), ("out", out), ("lse", lse), ("cu_q", cu_q),
                     ("workspace", workspace)))
    pages, heads, page_size, d = _cache(cache)
    if q.dim() != 3 or q.shape[2] != d or out.shape != q.shape or not q.is_contiguous() or not out.is_contiguous():
        raise ValueError(f"q and out must be contiguous and share one [T,H,{d}] shape")
    if out.dtype != q.dtype:
        raise ValueError("q and out must share one dtype")
    T, H, dt = q.shape[0], q.shape[1], _dtype_code(q)
    if lse.dtype != torch.float32 or tuple(lse.shape) != (T, H) or not lse.is_contiguous():
        raise ValueError("lse must be contiguous float32 [T,H]")
    if tables.dim() != 2:
        raise ValueError("tables must be contiguous int32 [B,width]")
    B, width = tables.shape
    _ints("tables", tables, (B, width))
    _ints("lens", lens, (B,))
    if cu_q is not None:
        _ints("cu_q", cu_q, (B + 1,))
        if max_q is None:
            raise ValueError("cu_q needs max_q, the largest number of queries of a sequence")
    elif (B == 0 and T) or (B and T % B) or (B and max_q is not None and max_q != T // B):
        raise ValueError("without cu_q every sequence has T / B queries")
    if T == 0:
        return
    if cu_q is None:
        max_q = T // B
    _fit("kv4_attn", T, B, width, int(max_q), pages)
    st = _stream(stream, cache.device)
    need = kv4_attn_workspace(T, B, H, heads, d, page_size, width, max_q)
    if workspace is not None:
        if not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
            raise ValueError(f"workspace must be contiguous with {need} bytes")
    elif need:
        workspace = binding.scratch(need, st, cache.device)
    with torch.cuda.device(cache.device):
        rc = lib().kv4_attn(q.data_ptr(), cache.data_ptr(), tables.data_ptr(), lens.data_ptr(), _ptr(cu_q), out.data_ptr(), lse.data_ptr(),
                            T, B, H, heads, d, pages, page_size, width, int(max_q), int(bool(causal)), float(scale), dt, _ptr(workspace),
                            need if workspace is not None else 0, st)
    if rc != KV4_OK:
        raise Kv4Error(rc, "kv4_attn")
