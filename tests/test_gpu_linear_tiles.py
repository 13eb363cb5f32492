"""The linear layers' epilogue on every tile and behind every joining of ranges, and backward passes whose products are split, against the formulas in
64 bits."""
import pytest
import torch

from tests import linear_cases as cases
from tests.block_ref import DTYPES, TINY, U, act, act_grad, inside, same

pytestmark = pytest.mark.gpu
NAN = float("nan")


def values(g, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * sigma).to(dtype)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def close(got, want, bound, what):
    error = (got.double() - want).abs()
    assert torch.isfinite(error).all(), what
    worst = (error / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


def epilogues(M, K, N, rows_of_n, dtype):
    """All activations, with the biases' types, a residual of its own or out's memory, and pre, in turn; pre in whole lines where 64 divides N."""
    from paper_2403_16863_amd import linear
    g = generator(M + N + K)
    x = values(g, (M, K), dtype)
    w = values(g, (N, K), dtype, K ** -0.5).t() if rows_of_n else values(g, (K, N), dtype, K ** -0.5)
    z0, size0 = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    residual = values(g, (M, N), dtype)
    for i, kind in enumerate(("none", "relu", "silu", "gelu", "gelu_tanh")):
        bias = [values(g, (N,), dtype), values(g, (N,), torch.float32), None][i % 3]
        form = ("apart", "in place", "none")[i % 3 if kind != "gelu" else 1]
        out, whole = inside((M, N), dtype, NAN, (2, 40))
        pre, whole_pre = inside((M, N), dtype, NAN, (1, 64)) if i != 2 else (None, None)
        if form == "in place":
            out.copy_(residual)
        linear.gemm_linear(x, w, out, bias, {"apart": residual, "in place": out, "none": None}[form], pre, kind)
        z, size = (z0, size0) if bias is None else (z0 + bias.double(), size0 + bias.double().abs())
        want = act(z, kind) + (0 if form == "none" else residual.double())
        # K products and a few terms summed in 32 bits, under activations of slope 1.13 at most; the activations' own error, 2^-20 of |z|: gelu's polynomial is
        # good to 5e-7 of a tail of 1/2 at most, and an exponential whose argument t is two roundings off moves p (1 - p) |t| <= 0.33 by 2^-23 of it, its value and the
        # reciprocal being a step each; and the last sum's rounding
        sums = (K + 8) * 2.0 ** -24 * size
        close(out, want, U[dtype] * want.abs() + TINY[dtype] + 1.2 * sums + 2.0 ** -20 * z.abs() + 2.0 ** -22 * want.abs() + 2.0 ** -23 * act(z, kind).abs(), (kind, "out"))
        assert torch.isnan(whole[M:]).all() and torch.isnan(whole[:, N:]).all()
        if pre is not None:
            close(pre, z, U[dtype] * z.abs() + TINY[dtype] + sums, (kind, "pre"))
            assert torch.isnan(whole_pre[M:]).all() and torch.isnan(whole_pre[:, N:]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tile,M,K,N,rows_of_n", cases.ON_TILES)
def test_epilogue_on_every_tile(tile, M, K, N, rows_of_n, dtype):
    from paper_2403_16863_amd import linear
    assert linear.linear_choice(M, N, K, linear.ROWS_N if rows_of_n else linear.ROWS) == (tile, 1)
    epilogues(M, K, N, rows_of_n, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,rows_of_n", cases.IN_RANGES)
def test_epilogue_behind_joined_ranges(M, K, N, rows_of_n, dtype):
    from paper_2403_16863_amd import linear
    assert linear.linear_choice(M, N, K, linear.ROWS_N if rows_of_n else linear.ROWS)[1] > 1
    epilogues(M, K, N, rows_of_n, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["none", "gelu"])
@pytest.mark.parametrize("M,N,K,w_rows,dw_rows", cases.BACKWARD_IN_RANGES)
def test_backward_with_both_sums_split(M, N, K, w_rows, dw_rows, kind, dtype):
    """A workspace of just the bytes asked for, between two others' memory: dz, the chunks' sums for dbias and the ranges' parts side by side in it, the parts of dx
    and then those of dw in the same place."""
    from paper_2403_16863_amd import linear
    g = generator(M + N)
    x, dy = values(g, (M, K), dtype), values(g, (M, N), dtype)
    w = values(g, (N, K), dtype, K ** -0.5).t() if w_rows else values(g, (K, N), dtype, K ** -0.5)
    pre = values(g, (M, N), dtype) if kind != "none" else None
    need, guard = linear.gemm_linear_bwd_workspace(M, N, K, kind, w_rows, dw_rows), 4096
    memory = torch.full((need + 2 * guard,), 255, dtype=torch.uint8, device="cuda")                # NaN
    got = []
    for workspace in (memory[guard:guard + need], None):
        dx, dw, dbias = torch.full_like(x, NAN), torch.full((N, K) if dw_rows else (K, N), NAN, dtype=dtype, device="cuda"), torch.full((N,), NAN, device="cuda")
        linear.gemm_linear_bwd(dy, x, w, pre, dx, dw.t() if dw_rows else dw, dbias, kind, workspace=workspace)
        got.append((dx, dw, dbias))
    assert (memory[:guard] == 255).all() and (memory[guard + need:] == 255).all()
    assert all(same(a, b) for a, b in zip(*got))
    dx, dw, dbias = got[0]
    dw = dw.t() if dw_rows else dw
    dz = dy.double() if pre is None else act_grad(pre.double(), kind, dy.double())
    # The kernel's dz is within 2^-18 of |dy| (gelu's slope: its polynomial 5e-7, its density's argument two roundings), and rounded once where there is an
    # activation: to a neighbouring number where a border between two is as near as that
    own = 2.0 ** -18 * dy.double().abs() * (pre is not None)
    rounded = dz.to(dtype).double()
    border = (dz + own).to(dtype).double() - (dz - own).to(dtype).double()
    x64, w64 = x.double(), w.double()
    for name, out, want, size, error, n in (("dx", dx, rounded @ w64.t(), rounded.abs() @ w64.abs().t(), border @ w64.abs().t(), N),
                                            ("dw", dw, x64.t() @ rounded, x64.abs().t() @ rounded.abs(), x64.abs().t() @ border, M)):
        close(out, want, U[dtype] * want.abs() + TINY[dtype] + (n + 8) * 2.0 ** -24 * size + error, name)
    close(dbias, dz.sum(0), (M + 8) * 2.0 ** -24 * dz.abs().sum(0) + own.sum(0) + 1e-30, "dbias")
