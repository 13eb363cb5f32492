"""Thin ctypes binding over the C ABI declared in include/linear.h: the matrix product with bias, activation and residual in its
epilogue, and its backward pass.

Argument marshalling only: every step runs in the HIP kernels of libattn.so.  There is no fallback: if the library
has not been built, loading it fails loudly.
"""
from __future__ import annotations

import ctypes

from . import binding

LINEAR_F16, LINEAR_BF16 = 0, 1
LINEAR_OK, LINEAR_EINVAL, LINEAR_EUNSUPPORTED, LINEAR_ELAUNCH, LINEAR_ENOMEM = 0, -1, -2, -3, -4
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
ROWS, ROWS_N, TOKENS = 0, 1, 2      # layouts of linear_product

# every symbol include/linear.h declares
SYMBOLS = ("gemm_linear", "gemm_linear_with", "gemm_linear_workspace", "gemm_linear_bwd", "gemm_linear_bwd_with", "gemm_linear_bwd_workspace",
           "linear_product", "linear_num_tiles", "linear_choice", "linear_strerror")

SCRATCH_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_void_p, ctypes.c_longlong)  # linear_scratch_fn


class Rows(ctypes.Structure):  # linear_rows
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_longlong)]


_ready = False


def lib():
    global _ready
    L = binding.lib()
    if not _ready:
        vp, i, ll, r, ip = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.POINTER(Rows), ctypes.POINTER(ctypes.c_int)
        L.gemm_linear.restype = i
        L.gemm_linear.argtypes = [r, r, i, vp, i, r, r, r, i, i, i, i, i, vp, ll, vp]
        L.gemm_linear_with.restype = i
        L.gemm_linear_with.argtypes = [r, r, i, vp, i, r, r, r, i, i, i, i, i, SCRATCH_FN, vp, vp]
        L.gemm_linear_bwd_with.restype = i
        L.gemm_linear_bwd_with.argtypes = [r, r, r, i, r, r, r, i, vp, i, i, i, i, i, SCRATCH_FN, vp, vp]
        L.gemm_linear_workspace.restype = ll
        L.gemm_linear_workspace.argtypes = [i] * 4
        L.gemm_linear_bwd.restype = i
        L.gemm_linear_bwd.argtypes = [r, r, r, i, r, r, r, i, vp, i, i, i, i, i, vp, ll, vp]
        L.gemm_linear_bwd_workspace.restype = ll
        L.gemm_linear_bwd_workspace.argtypes = [i] * 9
        L.linear_product.restype = i
        L.linear_product.argtypes = [r, r, i, r, i, i, i, i, i, i, vp, ll, vp]
        L.linear_num_tiles.restype = i
        L.linear_num_tiles.argtypes = []
        L.linear_choice.restype = i
        L.linear_choice.argtypes = [i, i, i, i, ip, ip]
        L.linear_strerror.restype = ctypes.c_char_p
        L.linear_strerror.argtypes = [i]
        _ready = True
    return L


def linear_strerror(code: int) -> str:
    return lib().linear_strerror(int(code)).decode()


class LinearError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {linear_strerror(code)} (code {code})")
        self.code = code


def _fit(what, *sizes):
    """The library counts in 32 bits, and ctypes would cut a larger number to them."""
    if max(sizes) > 2 ** 31 - 1 or min(sizes) < -2 ** 31:
        raise LinearError(LINEAR_EUNSUPPORTED, what)


def _activation(name):
    if name is None:
        return 0
    if name not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(ACTIVATIONS)}, got {name!r}")
    return ACTIVATIONS[name]


def _matrix(name, t, shape, like):
    if t is None:
        return
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if t.device != like.device:
        raise ValueError(f"{name} must live on the device of the other tensors")
    if t.dtype != like.dtype:
        raise ValueError(f"{name} must have the type of the other matrices, {like.dtype}, got {t.dtype}")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _rows(name, t):
    """A matrix with contiguous columns."""
    if t is None:
        return Rows(None, 0)
    if t.stride(1) != 1:
        raise ValueError(f"the columns of {name} must be contiguous")
    return Rows(t.data_ptr(), t.stride(0))


def _weight(name, t):
    """(Rows, rows_of_n) of a [K,N] matrix with contiguous columns, or the transposed view of an [N,K] one."""
    if t is None:
        return Rows(None, 0), 0
    if t.stride(1) == 1:
        return Rows(t.data_ptr(), t.stride(0)), 0
    if t.stride(0) == 1:
        return Rows(t.data_ptr(), t.stride(1)), 1
    raise ValueError(f"{name} must have contiguous columns, or be the transposed view of a matrix that has")


def _stream(stream, device):
    import torch
    return torch.cuda.current_stream(device).cuda_stream if stream is None else stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype(like):
    import torch
    if like.dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"matrices must be float16 or bfloat16, got {like.dtype}")
    return int(like.dtype == torch.bfloat16)


def _first(name):
    """The native module's function of that name, from the first call on (one lookup a call)."""
    def first(*args):
        lib()
        globals()["_plain_" + name] = call = getattr(binding.native(), "gemm_" + name)
        return call(*args)
    return first


_plain_linear, _plain_linear_bwd = _first("linear"), _first("linear_bwd")


def gemm_linear(x, w, out, bias=None, residual=None, pre=None, activation: str = "none", workspace=None, stream=None) -> None:
    """out <- act(x @ w + bias) + residual, and pre <- x @ w + bias where it is given (what the backward pass needs with an activation), for
    device tensors x [M,K], w [K,N], out, residual and pre [M,N], all float16 or all bfloat16, and bias [N] of that type or float32.  The
    columns of a matrix are contiguous and its rows have any stride that divides by 8; w may also be the transposed view `.t()` of a
    weight [N,K].  N and K divide by 8.  residual may be out itself.  activation: "none", "relu", "silu", "gelu" or "gelu_tanh".  Nothing is
    recorded for autograd: gemm_linear_bwd gives the gradients.
    Asynchronous on `stream` (an integer hipStream_t; default: torch's current stream).  Few tiles and a long K take scratch memory: `workspace`
    (uint8, gemm_linear_workspace bytes), or, on torch's current stream, memory of torch's allocator (the graph's own pool while torch records
    one); other streams and recordings do without."""
    rc = _plain_linear(x, w, out, bias, residual, pre, activation, workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise LinearError(rc, "gemm_linear")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[0]:
        raise ValueError("x must be [M,K] and w [K,N]")
    (M, K), N, dt, act = x.shape, w.shape[1], _dtype(x), _activation(activation)
    for name, t, shape in (("x", x, (M, K)), ("w", w, (K, N)), ("out", out, (M, N)), ("residual", residual, (M, N)), ("pre", pre, (M, N))):
        _matrix(name, t, shape, x)
    if out is None:
        raise ValueError("out must be given")
    f32 = _bias(bias, N, x)
    _fit("gemm_linear", M, N, K)
    (wr, rows_of_n), st = _weight("w", w), _stream(stream, x.device)
    rows = [_rows(name, t) for name, t in (("x", x), ("residual", residual), ("pre", pre), ("out", out))]
    need = gemm_linear_workspace(M, N, K, bool(rows_of_n))
    if workspace is not None:
        _check_workspace(workspace, need, x)
    elif need:
        workspace = binding.scratch(need, st, x.device)
    with torch.cuda.device(x.device):
        rc = lib().gemm_linear(rows[0], wr, rows_of_n, _ptr(bias), f32, rows[1], rows[2], rows[3], act, M, N, K, dt,
                               _ptr(workspace) if need else None, need if workspace is not None else 0, st)
    if rc != LINEAR_OK:
        raise LinearError(rc, "gemm_linear")


def _bias(bias, N, like):
    import torch
    if bias is None:
        return 0
    if not bias.is_cuda or bias.device != like.device:
        raise ValueError("bias must live on the device of the other tensors")
    if tuple(bias.shape) != (N,) or not bias.is_contiguous() or bias.dtype not in (like.dtype, torch.float32):
        raise ValueError("bias must be contiguous [N], float32 or of the matrices' type")
    return int(bias.dtype == torch.float32)


def _check_workspace(workspace, need, like):
    if not workspace.is_cuda or workspace.device != like.device:
        raise ValueError("workspace must live on the device of the other tensors")
    if not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"workspace must be contiguous with {need} bytes")


def gemm_linear_workspace(M: int, N: int, K: int, rows_of_n: bool = False) -> int:
    """Bytes of scratch memory that gemm_linear has a use for; rows_of_n: the weight is the transposed view of [N,K]."""
    sizes = [int(x) for x in (M, N, K)]
    _fit("gemm_linear_workspace", *sizes)
    n = lib().gemm_linear_workspace(*sizes, int(bool(rows_of_n)))
    if n < 0:
        raise LinearError(n, "gemm_linear_workspace")
    return n


def gemm_linear_bwd_workspace(M: int, N: int, K: int, activation: str = "none", rows_of_n: bool = False, dw_rows_of_n=None, dx: bool = True,
                              dw: bool = True, dbias: bool = True) -> int:
    """Bytes of scratch memory that gemm_linear_bwd needs for the gradients asked for; rows_of_n, dw_rows_of_n (default: the same): the weight, its
    gradient is the transposed view of [N,K]."""
    sizes = [int(x) for x in (M, N, K)]
    _fit("gemm_linear_bwd_workspace", *sizes)
    n = lib().gemm_linear_bwd_workspace(*sizes, int(bool(rows_of_n)), int(bool(rows_of_n if dw_rows_of_n is None else dw_rows_of_n)),
                                        _activation(activation), int(bool(dx)), int(bool(dw)), int(bool(dbias)))
    if n < 0:
        raise LinearError(n, "gemm_linear_bwd_workspace")
    return n


def gemm_linear_bwd(dy, x, w, pre=None, dx=None, dw=None, dbias=None, activation: str = "none", workspace=None, stream=None) -> None:
    """dx, dw, dbias <- gradients of gemm_linear from out's gradient dy [M,N]: dz = dy act'(pre), dx [M,K] = dz @ w.T, dw [K,N] = x.T @ dz,
    dbias (float32 [N]) = dz's sum over the rows.  Those that are None are left out, and so may be w without dx and x without dw; pre, the forward's,
    is needed with an activation.  dw may be the transposed view of [N,K], whichever w is.  With an activation dz is rounded to
    the matrices' type ahead of both products, and not for dbias.  The residual's gradient is dy itself.  All are written,
    none added to, and overlap nothing.
    The call needs scratch memory in most cases: `workspace` (uint8, gemm_linear_bwd_workspace bytes), or, on torch's current stream, memory that it
    takes from torch's allocator itself (the graph's own pool while torch records one).  On another stream, and in a recording begun
    elsewhere, the call is refused without the argument."""
    rc = _plain_linear_bwd(dy, x, w, pre, dx, dw, dbias, activation, workspace, stream)
    if not rc:
        return
    if rc < 0:
        raise LinearError(rc, "gemm_linear_bwd")
    # not a plain call: the steps one by one, each of which says what it refuses
    import torch
    if dx is None and dw is None and dbias is None:
        raise ValueError("one of dx, dw and dbias must be given")
    if dy.dim() != 2:
        raise ValueError("dy must be [M,N]")
    (M, N), dt, act = dy.shape, _dtype(dy), _activation(activation)
    if (dx is not None and w is None) or (dw is not None and x is None) or (act and pre is None):
        raise ValueError("dx needs w, dw needs x, and an activation needs pre")
    w, x, pre = w if dx is not None else None, x if dw is not None else None, pre if act else None
    first = dx if dx is not None else dw.t() if dw is not None else None
    if first is not None and first.dim() != 2:
        raise ValueError("gradients must be matrices")
    K = first.shape[1] if first is not None else 8       # (dbias alone: no product)
    for name, t, shape in (("dy", dy, (M, N)), ("x", x, (M, K)), ("w", w, (K, N)), ("pre", pre, (M, N)), ("dx", dx, (M, K)), ("dw", dw, (K, N))):
        _matrix(name, t, shape, dy)
    if dbias is not None and (not dbias.is_cuda or dbias.device != dy.device or dbias.dtype != torch.float32 or tuple(dbias.shape) != (N,) or
                              not dbias.is_contiguous()):
        raise ValueError("dbias must be contiguous float32 [N] on the device of the other tensors")
    _fit("gemm_linear_bwd", M, N, K)
    (wr, rows_of_n), (dwr, dw_rows_of_n), st = _weight("w", w), _weight("dw", dw), _stream(stream, dy.device)
    rows = [_rows(name, t) for name, t in (("dy", dy), ("x", x), ("pre", pre), ("dx", dx))]
    need = lib().gemm_linear_bwd_workspace(M, N, K, rows_of_n, dw_rows_of_n, act, dx is not None, dw is not None, dbias is not None)
    if need < 0:
        raise LinearError(need, "gemm_linear_bwd")
    if workspace is not None:
        _check_workspace(workspace, need, dy)
    elif need:
        workspace = binding.scratch(need, st, dy.device)
        if workspace is None:
            raise ValueError("a stream that is not torch's current one, or a recording that torch did not begin, needs a workspace")
    with torch.cuda.device(dy.device):
        rc = lib().gemm_linear_bwd(rows[0], rows[1], wr, rows_of_n, rows[2], rows[3], dwr, dw_rows_of_n, _ptr(dbias), act, M, N, K, dt,
                                   _ptr(workspace) if need else None, need, st)
    if rc != LINEAR_OK:
        raise LinearError(rc, "gemm_linear_bwd")


def linear_num_tiles() -> int:
    return int(lib().linear_num_tiles())


def linear_choice(M: int, N: int, K: int, layout: int):
    """(tile, ranges of k) that the calls above choose for a product c [M,N] over K, with a workspace."""
    tile, ranges = ctypes.c_int(0), ctypes.c_int(0)
    _fit("linear_choice", M, N, K)
    rc = lib().linear_choice(int(M), int(N), int(K), int(layout), ctypes.byref(tile), ctypes.byref(ranges))
    if rc != LINEAR_OK:
        raise LinearError(rc, "linear_choice")
    return tile.value, ranges.value


def linear_product(a, b, layout: int, c, tile: int, ranges: int = 1, workspace=None, stream=None) -> None:
    """c [M,N] <- the product of a and b as they lie in memory on tile `tile` with k in `ranges` parts, for tests and measurement: a [M,K], b
    [K,N] (ROWS); a [M,K], b [N,K] (ROWS_N); a [K,M], b [K,N] (TOKENS).  ranges > 1: workspace of ranges * M * N * 4 bytes."""
    import torch
    if layout not in (ROWS, ROWS_N, TOKENS):
        raise ValueError("layout must be ROWS, ROWS_N or TOKENS")
    for name, t in (("a", a), ("b", b), ("c", c)):
        if t.dim() != 2:
            raise ValueError(f"{name} must be a matrix")
    (M, N), K = c.shape, a.shape[0 if layout == TOKENS else 1]
    _matrix("a", a, (K, M) if layout == TOKENS else (M, K), a)
    _matrix("b", b, (N, K) if layout == ROWS_N else (K, N), a)
    _matrix("c", c, (M, N), a)
    _fit("linear_product", M, N, K)
    rows = [_rows(name, t) for name, t in (("a", a), ("b", b), ("c", c))]
    if workspace is not None:
        _check_workspace(workspace, 0, a)       # (how much the ranges need, the library knows)
    with torch.cuda.device(a.device):
        rc = lib().linear_product(rows[0], rows[1], int(layout), rows[2], M, N, K, _dtype(a), int(tile), int(ranges), _ptr(workspace),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream, a.device))
    if rc != LINEAR_OK:
        raise LinearError(rc, "linear_product")
