"""Thin ctypes binding over the C ABI declared in include/residual_norm.h: the norms behind a block and ahead of the next with the
residual stream's update between them, forward and backward.

Argument marshalling only: every step runs in the HIP kernels of libattn.so.  There is no fallback: if the library
has not been built, loading it fails loudly.
"""
from __future__ import annotations

import ctypes

from . import binding

NORM_F16, NORM_BF16 = 0, 1
NORM_OK, NORM_EINVAL, NORM_EUNSUPPORTED, NORM_ELAUNCH = 0, -1, -2, -3

# every symbol include/residual_norm.h declares
SYMBOLS = ("residual_norm", "residual_norm_bwd", "residual_norm_bwd_workspace", "norm_strerror")


class Tokens(ctypes.Structure):  # norm_tokens
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_longlong), ("token_stride", ctypes.c_longlong)]


class Vectors(ctypes.Structure):  # norm_vectors
    _fields_ = [("gate", ctypes.c_void_p), ("gate_stride", ctypes.c_longlong), ("gate_f32", ctypes.c_int), ("post_weight", ctypes.c_void_p),
                ("pre_weight", ctypes.c_void_p), ("weight_f32", ctypes.c_int), ("alpha", ctypes.c_float), ("eps", ctypes.c_float)]


_ready = False


def lib():
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i, ll, t, v = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(Tokens), ctypes.POINTER(Vectors)
        L.residual_norm.restype = i
        L.residual_norm.argtypes = [t] * 4 + [v, i, i, i, i, vp]
        L.residual_norm_bwd.restype = i
        L.residual_norm_bwd.argtypes = [t] * 6 + [v, vp, vp, vp, i, i, i, i, vp, ll, vp]
        L.residual_norm_bwd_workspace.restype = ll
        L.residual_norm_bwd_workspace.argtypes = [i] * 4
        L.norm_strerror.restype = ctypes.c_char_p
        L.norm_strerror.argtypes = [i]
        _ready = True
    return L


def norm_strerror(code: int) -> str:
    return lib().norm_strerror(int(code)).decode()


class NormError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {norm_strerror(code)} (code {code})")
        self.code = code


def _fit(what, *sizes):
    """The library counts in 32 bits, and ctypes would cut a larger number to them."""
    if max(sizes) > 2 ** 31 - 1 or min(sizes) < -2 ** 31:
        raise NormError(NORM_EUNSUPPORTED, what)


def _check(name, t, like):
    if t is None:
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if t.device != like.device:
        raise ValueError(f"{name} must live on the device of the other tensors")
    if t.dtype != like.dtype:
        raise ValueError(f"{name} must have the type of the other tensors of tokens, {like.dtype}, got {t.dtype}")
    if t.dim() != 3 or t.shape != like.shape:
        raise ValueError(f"{name} must be [B,N,C] with the sizes of the other tensors")
    if t.stride(2) != 1:
        raise ValueError(f"the channels of {name} must be contiguous")


def _tokens(t):
    return Tokens(None, 0, 0) if t is None else Tokens(t.data_ptr(), t.stride(0), t.stride(1))


def _vector(name, t, shapes, like, types):
    if t is None:
        return
    if not t.is_cuda or t.device != like.device:
        raise ValueError(f"{name} must live on the device of the other tensors")
    if tuple(t.shape) not in shapes or t.stride(-1) != 1 or t.dtype not in types:
        raise ValueError(f"{name} must be {' or '.join(str(list(s)) for s in shapes)} with contiguous channels, of {' or '.join(str(x) for x in types)}")


def _vectors(like, gate, post_weight, pre_weight, alpha, eps):
    import torch
    if like.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"tensors of tokens must be float16 or bfloat16, got {like.dtype}")
    if like.dim() != 3:
        raise ValueError("tensors of tokens must be [B,N,C]")
    (B, _, C), types = like.shape, (like.dtype, torch.float32)
    _vector("gate", gate, ((C,), (B, C)), like, types)
    _vector("post_weight", post_weight, ((C,),), like, types)
    _vector("pre_weight", pre_weight, ((C,),), like, types)
    if post_weight is not None and pre_weight is not None and post_weight.dtype != pre_weight.dtype:
        raise ValueError("both weights must have one type")
    weight = post_weight if post_weight is not None else pre_weight
    stride = gate.stride(0) if gate is not None and gate.dim() == 2 else 0
    if gate is not None and gate.dim() == 2 and B == 1:
        stride = C                          # the stride of a size of 1 is not looked at
    elif gate is not None and gate.dim() == 2 and stride < C:
        raise ValueError("the rows of gate must not overlap")
    return Vectors(_ptr(gate), stride, int(gate is not None and gate.dtype == torch.float32), _ptr(post_weight), _ptr(pre_weight),
                   int(weight is not None and weight.dtype == torch.float32), float(alpha), float(eps)), int(like.dtype == torch.bfloat16)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream, device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _first(name):
    """The native module's function of that name, from the first call on (one lookup a call)."""
    def first(*args):
        lib()
        globals()["_plain_" + name] = call = getattr(binding.native(), name)
        return call(*args)
    return first


_plain_residual_norm, _plain_residual_norm_bwd = _first("residual_norm"), _first("residual_norm_bwd")


def residual_norm(x, h, y, z, gate=None, post_weight=None, pre_weight=None, alpha: float = 1.0, eps: float = 1e-6, stream=None) -> None:
    """y <- alpha x + gate u with u = post_weight h / rms(h) (without post_weight u = h), and z <- pre_weight y / rms(y): the stream behind a block
    whose result is h, and the next block's input, for device tensors [B,N,C], all float16 or all bfloat16, with any strides that divide by 8 and
    contiguous channels.  gate: [C], or [B,C] with one for each sequence, or None; weights: [C]; each float32 or of the tensors' type.  h None: y = x, y and
    the block's arguments are left out too, and z is the plain norm of x.  y or z (with pre_weight) may be None.  y may be x itself,
    and any output an input of the same strides.  Nothing is recorded for autograd: residual_norm_bwd gives the gradients.
    Asynchronous on `stream` (an integer hipStream_t; default: torch's current stream)."""
    rc = _plain_residual_norm(x, h, y, z, gate, post_weight, pre_weight, alpha, eps, stream)
    if not rc:
        return
    if rc < 0:
        raise NormError(rc, "residual_norm")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    if x is None or (y is None and z is None):
        raise ValueError("x, and one of y and z, must be given")
    if (z is None) != (pre_weight is None):
        raise ValueError("z and pre_weight go together")
    if h is None and (y is not None or gate is not None or post_weight is not None or alpha != 1):
        raise ValueError("without h there is no y, gate, post_weight or alpha")
    vectors, dt = _vectors(x, gate, post_weight, pre_weight, alpha, eps)
    for name, t in (("x", x), ("h", h), ("y", y), ("z", z)):
        _check(name, t, x)
    B, N, C = x.shape
    _fit("residual_norm", B, N, C)
    with torch.cuda.device(x.device):
        rc = lib().residual_norm(*(_tokens(t) for t in (x, h, y, z)), vectors, B, N, C, dt, _stream(stream, x.device))
    if rc != NORM_OK:
        raise NormError(rc, "residual_norm")


def residual_norm_bwd_workspace(B: int, N: int, C: int, by_sequence: bool = False) -> int:
    """Bytes of scratch memory that residual_norm_bwd needs where a vector's gradient is asked for; by_sequence: the gate is [B,C]."""
    sizes = [int(x) for x in (B, N, C)]
    _fit("residual_norm_bwd_workspace", *sizes)
    n = lib().residual_norm_bwd_workspace(*sizes, int(bool(by_sequence)))
    if n < 0:
        raise NormError(n, "residual_norm_bwd_workspace")
    return n


def residual_norm_bwd(dy, dz, y, h, dx, dh, gate=None, post_weight=None, pre_weight=None, dgate=None, dpost_weight=None, dpre_weight=None,
                      alpha: float = 1.0, eps: float = 1e-6, workspace=None, stream=None) -> None:
    """dx, dh, dgate, dpost_weight, dpre_weight <- gradients of residual_norm, from those of y and z (either may be None; dz goes with pre_weight), the
    forward's y (x, where there was no h; not needed without dz) and h (not needed without a gate and post_weight).  Gradients that are
    None are left out (dx or dh must be there); the vectors' are float32 with the vectors' shapes, contiguous, written.  With one of those the
    call needs scratch memory: `workspace` (uint8, residual_norm_bwd_workspace bytes), or, on torch's current stream,
    memory that it takes from torch's allocator itself (the graph's own pool while torch records one).  On another stream, and in
    a recording begun elsewhere, the call is refused without the argument.  dx may be dy itself, and dx and dh any input of the same strides."""
    rc = _plain_residual_norm_bwd(dy, dz, y, h, dx, dh, gate, post_weight, pre_weight, dgate, dpost_weight, dpre_weight, alpha, eps, workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise NormError(rc, "residual_norm_bwd")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    like = dy if dy is not None else dz
    if like is None or (dx is None and dh is None):
        raise ValueError("one of dy and dz, and one of dx and dh, must be given")
    if (dz is None) != (pre_weight is None) or (dz is not None and y is None):
        raise ValueError("dz goes with pre_weight, and needs the forward's y")
    if (gate is not None or post_weight is not None) and h is None:
        raise ValueError("a gate or post_weight needs the forward's h")
    for name, d, t in (("dgate", dgate, gate), ("dpost_weight", dpost_weight, post_weight), ("dpre_weight", dpre_weight, pre_weight)):
        if d is not None and t is None:
            raise ValueError(f"{name} has no vector")
    y, h = y if dz is not None else None, h if gate is not None or post_weight is not None else None
    vectors, dt = _vectors(like, gate, post_weight, pre_weight, alpha, eps)
    for name, t in (("dy", dy), ("dz", dz), ("y", y), ("h", h), ("dx", dx), ("dh", dh)):
        _check(name, t, like)
    B, N, C = like.shape
    _fit("residual_norm_bwd", B, N, C)
    for name, d, t in (("dgate", dgate, gate), ("dpost_weight", dpost_weight, post_weight), ("dpre_weight", dpre_weight, pre_weight)):
        if d is not None and (not d.is_cuda or d.device != like.device or d.dtype != torch.float32 or d.shape != t.shape or not d.is_contiguous()):
            raise ValueError(f"{name} must be contiguous float32 with its vector's shape, on the device of the other tensors")
    st, need = _stream(stream, like.device), 0
    if dgate is not None or dpost_weight is not None or dpre_weight is not None:
        need = residual_norm_bwd_workspace(B, N, C, vectors.gate_stride > 0)
        if workspace is None:
            workspace = binding.scratch(need, st, like.device)
            if workspace is None:
                raise ValueError("a stream that is not torch's current one, or a recording that torch did not begin, needs a workspace")
        elif not workspace.is_cuda or workspace.device != like.device:
            raise ValueError("workspace must live on the device of the other tensors")
        elif not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
            raise ValueError(f"workspace must be contiguous with {need} bytes")
    with torch.cuda.device(like.device):
        rc = lib().residual_norm_bwd(*(_tokens(t) for t in (dy, dz, y, h, dx, dh)), vectors, _ptr(dgate), _ptr(dpost_weight), _ptr(dpre_weight),
                                     B, N, C, dt, _ptr(workspace) if need else None, need, st)
    if rc != NORM_OK:
        raise NormError(rc, "residual_norm_bwd")
