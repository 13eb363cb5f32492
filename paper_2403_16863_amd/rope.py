"""Thin ctypes binding over the C ABI declared in include/qk_rope.h: norms of queries and keys for each head with the position
rotation in the same pass, forward and backward.

Argument marshalling only: every step runs in the HIP kernels of libattn.so.  There is no fallback: if the library
has not been built, loading it fails loudly.
"""
from __future__ import annotations

import ctypes

from . import binding

QK_F16, QK_BF16 = 0, 1
QK_OK, QK_EINVAL, QK_EUNSUPPORTED, QK_ELAUNCH = 0, -1, -2, -3

# every symbol include/qk_rope.h declares
SYMBOLS = ("qk_norm_rope", "qk_norm_rope_bwd", "qk_norm_rope_axes", "qk_norm_rope_axes_bwd", "qk_norm_rope_bwd_workspace", "qk_strerror")
NO_AXIS = 255


class Heads(ctypes.Structure):  # qk_heads
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_longlong), ("token_stride", ctypes.c_longlong),
                ("head_stride", ctypes.c_longlong)]


_ready = False


def lib():
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i, f, h = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.POINTER(Heads)
        L.qk_norm_rope.restype = i
        L.qk_norm_rope.argtypes = [h] * 4 + [vp, vp, i, vp, vp, vp, i, f] + [i] * 7 + [vp]
        L.qk_norm_rope_bwd.restype = i
        L.qk_norm_rope_bwd.argtypes = [h] * 6 + [vp, vp, i, vp, vp, vp, vp, vp, i, f] + [i] * 7 + [vp, ctypes.c_longlong, vp]
        L.qk_norm_rope_axes.restype = i
        L.qk_norm_rope_axes.argtypes = [h] * 4 + [vp, vp, i, vp, vp, vp, i, i, ctypes.c_char_p, f] + [i] * 7 + [vp]
        L.qk_norm_rope_axes_bwd.restype = i
        L.qk_norm_rope_axes_bwd.argtypes = [h] * 6 + [vp, vp, i, vp, vp, vp, vp, vp, i, i, ctypes.c_char_p, f] + [i] * 7 + [vp, ctypes.c_longlong, vp]
        L.qk_norm_rope_bwd_workspace.restype = ctypes.c_longlong
        L.qk_norm_rope_bwd_workspace.argtypes = [i] * 5
        L.qk_strerror.restype = ctypes.c_char_p
        L.qk_strerror.argtypes = [i]
        _ready = True
    return L


def qk_strerror(code: int) -> str:
    return lib().qk_strerror(int(code)).decode()


class RopeError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {qk_strerror(code)} (code {code})")
        self.code = code


def _fit(what, *sizes):
    """The library counts in 32 bits, and ctypes would cut a larger number to them."""
    if max(sizes) > 2 ** 31 - 1 or min(sizes) < -2 ** 31:
        raise RopeError(QK_EUNSUPPORTED, what)


def _check_heads(name, t, like, heads=None):
    if t is None:
        return
    if t.dim() != 4 or t.shape[0] != like.shape[0] or t.shape[1] != like.shape[1] or t.shape[3] != like.shape[3]:
        raise ValueError(f"{name} must be [B,N,heads,d] with the sizes of the other tensors")
    if heads is not None and t.shape[2] != heads:
        raise ValueError(f"{name} must have {heads} heads")
    if t.dtype != like.dtype:
        raise ValueError("queries, keys and their outputs or gradients must share one dtype")
    if t.stride(3) != 1:
        raise ValueError(f"the channels of {name} must be contiguous")


def _heads(t):
    return Heads(None, 0, 0, 0) if t is None else Heads(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _common(like, cos, sin, positions, weights, given, axes=None):
    import torch
    for name, t in given:
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{name} must live in device memory")
        if t.device != like.device:
            raise ValueError(f"{name} must live on the device of the other tensors")
    if like.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"queries and keys must be float16 or bfloat16, got {like.dtype}")
    B, N, _, d = like.shape
    if axes is None:
        if positions.dtype != torch.int32 or tuple(positions.shape) != (B, N) or not positions.is_contiguous():
            raise ValueError("positions must be contiguous int32 [B,N]")
    else:
        if positions.dtype != torch.int32 or positions.dim() != 3 or tuple(positions.shape[:2]) != (B, N) or not positions.is_contiguous():
            raise ValueError("positions must be contiguous int32 [B,N,axes]")
        if not isinstance(axes, bytes) or len(axes) != d // 2:
            raise ValueError(f"axes must be d/2 = {d // 2} bytes, one for each pair (axes_of_pairs makes them)")
        if not 1 <= positions.shape[2] <= 4 or any(a >= positions.shape[2] and a != NO_AXIS for a in axes):
            raise ValueError("positions must have 1 to 4 axes, and axes name one of them, or NO_AXIS, for each pair")
    for name, t in (("cos", cos), ("sin", sin)):
        if t.dtype != torch.float32 or t.dim() != 2 or t.shape[1] != d // 2 or t.shape != cos.shape or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous float32 [rows,d/2]")
    weights = [w for w in weights if w is not None]
    for w in weights:
        if tuple(w.shape) != (d,) or not w.is_contiguous() or w.dtype not in (like.dtype, torch.float32) or w.dtype != weights[0].dtype:
            raise ValueError("weights must be contiguous [d], both float32 or both of the type of queries and keys")
    return int(bool(weights) and weights[0].dtype == torch.float32), int(like.dtype == torch.bfloat16)


def _stream(stream, device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _first(name):
    """The native module's function of that name, from the first call on (one lookup a call)."""
    def first(*args):
        lib()
        globals()["_plain_" + name] = call = getattr(binding.native(), "qk_" + name)
        return call(*args)
    return first


_plain_norm_rope, _plain_norm_rope_bwd = _first("norm_rope"), _first("norm_rope_bwd")
_plain_norm_rope_axes, _plain_norm_rope_axes_bwd = _first("norm_rope_axes"), _first("norm_rope_axes_bwd")


def qk_norm_rope(q, k, q_out, k_out, cos, sin, positions, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                 stream=None) -> None:
    """q_out, k_out <- norm (where there is a weight) and rotation of q [B,N,H,d] and k [B,N,Hkv,d].  All four may have any
    strides that divide by 8 with contiguous channels: slices of a joint projection, or the transposed view of attn_fwd's [B,H,N,d];
    q or k may be None with its output.  cos, sin: float32 [rows,d/2]; positions: int32 [B,N].  Nothing is recorded for
    autograd: qk_norm_rope_bwd gives the gradients.  Asynchronous on `stream` (an integer hipStream_t; default: torch's current stream)."""
    rc = _plain_norm_rope(q, k, q_out, k_out, cos, sin, positions, q_weight, k_weight, eps, interleaved, stream)
    if not rc:
        return
    if rc < 0:
        raise RopeError(rc, "qk_norm_rope")
    _forward("qk_norm_rope", q, k, q_out, k_out, cos, sin, positions, None, q_weight, k_weight, eps, interleaved, stream)


def _forward(what, q, k, q_out, k_out, cos, sin, positions, axes, q_weight, k_weight, eps, interleaved, stream) -> None:
    """Not a plain call: the steps one by one, each of which says what it refuses."""
    import torch
    like = q if q is not None else k
    if like is None or (q is None) != (q_out is None) or (k is None) != (k_out is None):
        raise ValueError("q and q_out, k and k_out go together, and one pair must be there")
    H, Hkv = (0 if t is None else t.shape[2] if t.dim() == 4 else 0 for t in (q, k))
    for name, t, heads in (("q", q, None), ("k", k, None), ("q_out", q_out, H), ("k_out", k_out, Hkv)):
        _check_heads(name, t, like, heads)
    f32, dt = _common(like, cos, sin, positions, (q_weight, k_weight),
                      (("q", q), ("k", k), ("q_out", q_out), ("k_out", k_out), ("cos", cos), ("sin", sin), ("positions", positions),
                       ("q_weight", q_weight), ("k_weight", k_weight)), axes)
    B, N, _, d = like.shape
    _fit(what, B, N, H, Hkv, cos.shape[0])
    hs = [_heads(t) for t in (q, k, q_out, k_out)]
    by = () if axes is None else (positions.shape[2], axes)
    with torch.cuda.device(like.device):
        rc = getattr(lib(), what)(*hs, _ptr(q_weight), _ptr(k_weight), f32, cos.data_ptr(), sin.data_ptr(), positions.data_ptr(), cos.shape[0], *by,
                                  float(eps), int(bool(interleaved)), B, N, H, Hkv, d, dt, _stream(stream, like.device))
    if rc != QK_OK:
        raise RopeError(rc, what)


def axes_of_pairs(sections, d: int, alternating: bool = False) -> bytes:
    """The axis of each of the d/2 pairs, as qk_norm_rope_axes takes them: sections[a] pairs turn by axis a, one axis after the other or, alternating, the
    axes taking turns until their shares are used up; pairs behind the last are not turned."""
    left = [int(n) for n in sections]
    if not 1 <= len(left) <= 4 or min(left) < 0 or sum(left) > d // 2:
        raise ValueError(f"sections must be 1 to 4 numbers of pairs, {d // 2} in all at most")
    found = []
    if alternating:
        while any(left):
            for a, n in enumerate(left):
                if n:
                    found.append(a)
                    left[a] -= 1
    else:
        for a, n in enumerate(left):
            found += [a] * n
    return bytes(found + [NO_AXIS] * (d // 2 - len(found)))


def qk_norm_rope_axes(q, k, q_out, k_out, cos, sin, positions, axes, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                      stream=None) -> None:
    """qk_norm_rope with positions on several axes, int32 [B,N,axes] with 1 to 4 of them (time, height and width of a video's patches, say): each pair of
    channels turns by the row of cos and sin that the position on its own axis names.  axes: the axis of each of the d/2 pairs, as bytes
    (axes_of_pairs makes them), NO_AXIS for a pair that is not turned."""
    rc = _plain_norm_rope_axes(q, k, q_out, k_out, cos, sin, positions, axes, q_weight, k_weight, eps, interleaved, stream)
    if not rc:
        return
    if rc < 0:
        raise RopeError(rc, "qk_norm_rope_axes")
    _forward("qk_norm_rope_axes", q, k, q_out, k_out, cos, sin, positions, axes, q_weight, k_weight, eps, interleaved, stream)


def qk_norm_rope_bwd_workspace(B: int, N: int, H: int, Hkv: int, d: int) -> int:
    """Bytes of scratch memory that qk_norm_rope_bwd needs where there is a weight."""
    sizes = [int(x) for x in (B, N, H, Hkv, d)]
    _fit("qk_norm_rope_bwd_workspace", *sizes)
    n = lib().qk_norm_rope_bwd_workspace(*sizes)
    if n < 0:
        raise RopeError(n, "qk_norm_rope_bwd_workspace")
    return n


def qk_norm_rope_bwd(dq_out, dk_out, q, k, dq, dk, cos, sin, positions, q_weight=None, k_weight=None, dq_weight=None, dk_weight=None,
                     eps: float = 1e-6, interleaved: bool = False, workspace=None, stream=None) -> None:
    """dq, dk, dq_weight, dk_weight <- gradients of qk_norm_rope, from those of its outputs and its inputs q, k (not needed, and
    None will do, for a tensor without a weight).  dq_weight, dk_weight: float32 [d], written.  With a weight
    the call needs scratch memory: `workspace` (uint8, qk_norm_rope_bwd_workspace bytes), or, on torch's current stream,
    memory that it takes from torch's allocator itself (the graph's own pool while torch records one).  On another stream, and in
    a recording begun elsewhere, the call is refused without the argument."""
    rc = _plain_norm_rope_bwd(dq_out, dk_out, q, k, dq, dk, cos, sin, positions, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved,
                              workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise RopeError(rc, "qk_norm_rope_bwd")
    _backward("qk_norm_rope_bwd", dq_out, dk_out, q, k, dq, dk, cos, sin, positions, None, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved,
              workspace, stream)


def _backward(what, dq_out, dk_out, q, k, dq, dk, cos, sin, positions, axes, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved, workspace,
              stream) -> None:
    """Not a plain call: the steps one by one, each of which says what it refuses."""
    import torch
    like = dq_out if dq_out is not None else dk_out
    if like is None or (dq_out is None) != (dq is None) or (dk_out is None) != (dk is None):
        raise ValueError("dq_out and dq, dk_out and dk go together, and one pair must be there")
    if (q_weight is None) != (dq_weight is None) or (k_weight is None) != (dk_weight is None):
        raise ValueError("a weight and its gradient go together")
    if (q_weight is not None and (q is None or dq is None)) or (k_weight is not None and (k is None or dk is None)):
        raise ValueError("a tensor with a weight needs the forward's input")
    H, Hkv = (0 if t is None else t.shape[2] if t.dim() == 4 else 0 for t in (dq_out, dk_out))
    q, k = q if q_weight is not None else None, k if k_weight is not None else None
    for name, t, heads in (("dq_out", dq_out, None), ("dk_out", dk_out, None), ("q", q, H), ("k", k, Hkv), ("dq", dq, H), ("dk", dk, Hkv)):
        _check_heads(name, t, like, heads)
    f32, dt = _common(like, cos, sin, positions, (q_weight, k_weight),
                      (("dq_out", dq_out), ("dk_out", dk_out), ("q", q), ("k", k), ("dq", dq), ("dk", dk), ("cos", cos), ("sin", sin),
                       ("positions", positions), ("q_weight", q_weight), ("k_weight", k_weight), ("dq_weight", dq_weight),
                       ("dk_weight", dk_weight), ("workspace", workspace)), axes)
    B, N, _, d = like.shape
    _fit(what, B, N, H, Hkv, cos.shape[0])
    for w in (dq_weight, dk_weight):
        if w is not None and (w.dtype != torch.float32 or tuple(w.shape) != (d,) or not w.is_contiguous()):
            raise ValueError("gradients of weights must be contiguous float32 [d]")
    st, need = _stream(stream, like.device), 0
    hs = [_heads(t) for t in (dq_out, dk_out, q, k, dq, dk)]
    if q_weight is not None or k_weight is not None:
        need = qk_norm_rope_bwd_workspace(B, N, H, Hkv, d)
        if workspace is None:
            workspace = binding.scratch(need, st, like.device)
            if workspace is None:
                raise ValueError("a stream that is not torch's current one, or a recording that torch did not begin, needs a workspace")
        elif not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
            raise ValueError(f"workspace must be contiguous with {need} bytes")
    by = () if axes is None else (positions.shape[2], axes)
    with torch.cuda.device(like.device):
        rc = getattr(lib(), what)(*hs, _ptr(q_weight), _ptr(k_weight), f32, _ptr(dq_weight), _ptr(dk_weight), cos.data_ptr(), sin.data_ptr(),
                                  positions.data_ptr(), cos.shape[0], *by, float(eps), int(bool(interleaved)), B, N, H, Hkv, d, dt,
                                  _ptr(workspace) if need else None, need, st)
    if rc != QK_OK:
        raise RopeError(rc, what)


def qk_norm_rope_axes_bwd(dq_out, dk_out, q, k, dq, dk, cos, sin, positions, axes, q_weight=None, k_weight=None, dq_weight=None, dk_weight=None,
                          eps: float = 1e-6, interleaved: bool = False, workspace=None, stream=None) -> None:
    """The gradients of qk_norm_rope_axes, as qk_norm_rope_bwd gives those of qk_norm_rope (its workspace is the same)."""
    rc = _plain_norm_rope_axes_bwd(dq_out, dk_out, q, k, dq, dk, cos, sin, positions, axes, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved,
                                   workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise RopeError(rc, "qk_norm_rope_axes_bwd")
    _backward("qk_norm_rope_axes_bwd", dq_out, dk_out, q, k, dq, dk, cos, sin, positions, axes, q_weight, k_weight, dq_weight, dk_weight, eps, interleaved,
              workspace, stream)
