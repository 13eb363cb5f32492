"""A transformer block of the framework's operators, as a model runs them: forward with the attention between, backward behind the attention, and
steps of single tokens."""
import pytest
import torch

from tests.block_ref import DTYPES, U, act, rms, same

pytestmark = pytest.mark.gpu


def weights(dtype, C, H, Hkv, d, hidden, seed=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return (torch.randn(*shape, generator=g) * sigma).to(dtype).cuda()
    return dict(norm1=torch.rand(C, generator=g).add(0.5).cuda(), post=torch.rand(C, generator=g).add(0.5).cuda(), norm2=torch.rand(C, generator=g).add(0.5).cuda(),
                qw=torch.rand(d, generator=g).add(0.5).to(dtype).cuda(), kw=torch.rand(d, generator=g).add(0.5).to(dtype).cuda(),
                qkv=normal((H + 2 * Hkv) * d, C, sigma=C ** -0.5).t(), qkv_bias=normal((H + 2 * Hkv) * d, sigma=0.1),
                out=normal(H * d, C, sigma=(H * d) ** -0.5), up=normal(hidden, C, sigma=C ** -0.5).t(), up_bias=normal(hidden, sigma=0.1),
                down=normal(hidden, C, sigma=hidden ** -0.5), down_bias=normal(C, sigma=0.1).float())


def block(w, x, gate, cos, sin, positions, axes, H, d, keep=None):
    """The block's output for a stream x [B,N,C]; keep: a dict for what the backward pass needs."""
    import paper_2403_16863_amd as A
    from paper_2403_16863_amd import linear, norm, rope
    B, N, C = x.shape

    def new(*shape):
        return torch.empty(*shape, dtype=x.dtype, device="cuda")
    z, qkv = new(B, N, C), new(B * N, w["qkv"].shape[1])
    norm.residual_norm(x, None, None, z, None, None, w["norm1"])
    linear.gemm_linear(z.view(B * N, C), w["qkv"], qkv, w["qkv_bias"])
    heads = qkv.view(B, N, 3 * H, d)
    q, k, o, lse = new(B, H, N, d), new(B, H, N, d), new(B, H, N, d), torch.empty(B, H, N, device="cuda")
    rope.qk_norm_rope_axes(heads[:, :, :H], heads[:, :, H:2 * H], q.transpose(1, 2), k.transpose(1, 2), cos, sin, positions, axes, w["qw"], w["kw"])
    A.attn_fwd(q, k, heads[:, :, 2 * H:].transpose(1, 2).contiguous(), o, lse, False, d ** -0.5)
    a = new(B * N, C)
    linear.gemm_linear(o.transpose(1, 2).reshape(B * N, H * d), w["out"], a)
    y, z2 = new(B, N, C), new(B, N, C)
    norm.residual_norm(x, a.view(B, N, C), y, z2, gate, w["post"], w["norm2"])
    hidden, pre, out = new(B * N, w["up"].shape[1]), new(B * N, w["up"].shape[1]), new(B * N, C)
    linear.gemm_linear(z2.view(B * N, C), w["up"], hidden, w["up_bias"], None, pre, "gelu_tanh")
    linear.gemm_linear(hidden, w["down"], out, w["down_bias"], y.view(B * N, C))
    if keep is not None:
        keep.update(a=a.view(B, N, C), y=y, z2=z2, hidden=hidden, pre=pre)
    return out.view(B, N, C)


def second_half_64(w, x, a, gate):
    """From the attention's projection on, differentiable."""
    post, norm2 = w["post"], w["norm2"]
    y = x + gate[:, None] * (post * a * rms(a, 1e-6))
    z2 = norm2 * y * rms(y, 1e-6)
    return y + act(z2 @ w["up"] + w["up_bias"], "gelu_tanh") @ w["down"] + w["down_bias"]


def block_64(w, x, gate, cos, sin, positions, axes, H, d):
    B, N, C = x.shape
    z = w["norm1"] * x * rms(x, 1e-6)
    heads = (z @ w["qkv"] + w["qkv_bias"]).view(B, N, 3 * H, d)
    co, si = torch.ones(B, N, 1, d // 2, device="cuda", dtype=torch.float64), torch.zeros(B, N, 1, d // 2, device="cuda", dtype=torch.float64)
    for p, axis in enumerate(axes):
        if axis != 255:
            at = positions[..., axis].long()
            co[:, :, 0, p], si[:, :, 0, p] = cos.double()[at, p], sin.double()[at, p]

    def turn(v, weight):
        v = v * rms(v, 1e-6) * weight
        m, n = v.chunk(2, -1)
        return torch.cat((m * co - n * si, n * co + m * si), -1).transpose(1, 2).contiguous()
    q, k, v = turn(heads[:, :, :H], w["qw"]), turn(heads[:, :, H:2 * H], w["kw"]), heads[:, :, 2 * H:].transpose(1, 2).contiguous()
    p = torch.softmax(q @ k.transpose(2, 3).contiguous() * d ** -0.5, -1)
    a = (p @ v).transpose(1, 2).reshape(B, N, H * d) @ w["out"]
    return a, second_half_64(w, x, a, gate)


def setup(dtype, B=2, T=2, Y=5, X=7, C=264, H=3, d=64, hidden=1032):
    from paper_2403_16863_amd import rope
    w, N = weights(dtype, C, H, H, d, hidden), T * Y * X
    g = torch.Generator().manual_seed(3)
    x, gate = torch.randn(B, N, C, generator=g).to(dtype).cuda(), torch.randn(B, C, generator=g).to(dtype).cuda()
    n = torch.arange(N)
    positions = torch.stack((n // (Y * X), n // X % Y, n % X), -1).expand(B, N, 3).int().contiguous().cuda()
    angle = torch.arange(16, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    return w, x, gate, angle.cos().float().cuda(), angle.sin().float().cuda(), positions, rope.axes_of_pairs((8, 12, 12), d), H, d


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", DTYPES)
def test_block_forward_and_backward(dtype):
    from paper_2403_16863_amd import linear, norm
    args, kept = setup(dtype), {}
    w, x, gate = args[:3]
    out = block(*args, keep=kept)
    w64 = {k: v.double() for k, v in w.items()}
    _, want = block_64(w64, x.double(), gate.double(), *args[3:])
    # Eleven tensors are rounded on the way (z, qkv, q, k, the probabilities, o, a, y, z2, hidden, out), each by half a step at most, 0.58 of it in the
    # mean square, and each of the steps behind keeps a relative error within about twice its size (norms and softmax of scores of a few units)
    assert off(out, want) <= 2 * 11 ** 0.5 * U[dtype]

    B, N, C = x.shape
    g = torch.Generator().manual_seed(4)
    dout = torch.randn(B, N, C, generator=g).to(dtype).cuda()
    rows = dout.view(B * N, C)

    def grads():
        """The second half's gradients, from the output's."""
        t = {k: torch.empty_like(v) for k, v in (("down", w["down"]), ("up", w["up"]), ("hidden", kept["hidden"]), ("z2", kept["z2"]), ("dx", x), ("da", x))}
        f = {k: torch.empty(v.shape, device="cuda") for k, v in (("down_bias", w["down_bias"]), ("up_bias", w["up_bias"]), ("gate", gate), ("post", w["post"]),
                                                                ("norm2", w["norm2"]))}
        linear.gemm_linear_bwd(rows, kept["hidden"], w["down"], None, t["hidden"], t["down"], f["down_bias"])
        linear.gemm_linear_bwd(t["hidden"], kept["z2"].view(B * N, C), w["up"], kept["pre"], t["z2"].view(B * N, C), t["up"], f["up_bias"], "gelu_tanh")
        norm.residual_norm_bwd(dout, t["z2"], kept["y"], kept["a"], t["dx"], t["da"], gate, w["post"], w["norm2"], f["gate"], f["post"], f["norm2"])
        return {**t, **{"f_" + k: v for k, v in f.items()}}
    got = grads()
    leaves = {k: v.clone().requires_grad_() for k, v in {**w64, "x": x.double(), "a": kept["a"].double(), "gate64": gate.double()}.items()}
    second_half_64(leaves, leaves["x"], leaves["a"], leaves["gate64"]).backward(dout.double())
    names = {"down": "down", "up": "up", "dx": "x", "da": "a", "f_down_bias": "down_bias", "f_up_bias": "up_bias", "f_gate": "gate64", "f_post": "post", "f_norm2": "norm2"}
    for mine, leaf in names.items():
        # at most eight roundings (y, z2, pre, hidden forward; dhidden, dz, dz2 and the result backward), as above
        assert off(got[mine], leaves[leaf].grad) <= 2 * 8 ** 0.5 * U[dtype], mine
    again = grads()
    assert all(same(got[k], again[k]) for k in got)


def test_block_in_a_graph():
    """The whole run recorded and replayed, with eager runs between, gives the eager run's bits."""
    args = setup(torch.bfloat16)
    want = block(*args)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(*args)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        out = block(*args)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, want) and same(block(*args), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_single_tokens_match_the_rows_of_a_prompt(dtype):
    """The operators around the attention for one token at a time: rows of the same calls on all of them, to the rounding of sums in another order."""
    from paper_2403_16863_amd import linear, norm
    C, hidden, N = 264, 1032, 9
    w = weights(dtype, C, 2, 2, 64, hidden)
    g = torch.Generator().manual_seed(5)
    x, h = (torch.randn(1, N, C, generator=g).to(dtype).cuda() for _ in range(2))

    def run(x, h):
        n = x.shape[1]
        y, z, up, out = torch.empty_like(x), torch.empty_like(x), torch.empty(n, hidden, dtype=dtype, device="cuda"), torch.empty(n, C, dtype=dtype, device="cuda")
        norm.residual_norm(x, h, y, z, None, w["post"], w["norm2"])
        linear.gemm_linear(z[0], w["up"], up, w["up_bias"], activation="silu")
        linear.gemm_linear(up, w["down"], out, w["down_bias"], y[0])
        return y, z, out
    y, z, out = run(x, h)
    for i in range(N):
        y1, z1, out1 = run(x[:, i:i + 1], h[:, i:i + 1])
        assert same(y1, y[:, i:i + 1]) and same(z1, z[:, i:i + 1])     # a token's sums are its own
        # hidden may be rounded the other way in a few places: a step of each at most, and one of the result
        size = up_size = w["down"].double().abs().sum(0).max().item() * 4
        assert (out1.double() - out[i:i + 1].double()).abs().max().item() <= 2 * U[dtype] * (size + out.double().abs().max().item()) * 1.0 and up_size > 0
