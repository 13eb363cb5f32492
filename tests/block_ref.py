"""The operators around the attention forward in 64 bits, on the device of their inputs: linear layers' epilogue, the norms with the
residual stream, and helpers of their tests."""
import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half a step of the smallest numbers
DTYPES = [torch.float16, torch.bfloat16]


def act(z, kind):
    """The gelus in forms that keep their digits for negative z, where 1 + erf and 1 + tanh end at 2^-53: 1 + erf(x) = erfc(-x), and
    1 + tanh(u) = 2 / (1 + e^-2u)."""
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z * 0.5 ** 0.5)
    if kind == "gelu_tanh":
        return z * torch.sigmoid((8 / torch.pi) ** 0.5 * (z + 0.044715 * z * z * z))
    return {"none": lambda v: v * 1, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v)}[kind](z)


def act_grad(z, kind, dy):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act(z, kind), z, dy)[0]


def rms(v, eps):
    return (v.pow(2).mean(-1, keepdim=True) + eps).rsqrt()


def per_token(gate):
    return 1.0 if gate is None else gate[:, None] if gate.dim() == 2 else gate


def residual_norm(x, h, gate, post, pre, alpha, eps):
    y = x
    if h is not None:
        u = h if post is None else post * h * rms(h, eps)
        y = alpha * x + per_token(gate) * u
    return y, None if pre is None else pre * y * rms(y, eps)


def inside(shape, dtype, fill, more=(1, 8), device="cuda"):
    """A view of that shape inside a larger tensor of `fill`: (view, whole).  more: what the last dimensions are longer by."""
    wide = list(shape)
    for i, n in enumerate(more):
        wide[len(shape) - len(more) + i] += n
    whole = torch.full(wide, fill, dtype=dtype, device=device)
    view = whole
    for i, n in enumerate(shape):
        view = view.narrow(i, 0, n)
    return view, whole


def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def same(a, b):
    return torch.equal(bits(a), bits(b))
