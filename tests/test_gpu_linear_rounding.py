"""What the gradients of a linear layer with an activation are rounded by: dz to the matrices' type, ahead of both products, and the result, each
once, and nothing else."""
import pytest
import torch

from tests.block_ref import DTYPES, TINY, U, act_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("M,N,K", [(300, 520, 264), (1001, 1032, 200)])
def test_gradients_are_products_of_dz_rounded_once(M, N, K, kind, dtype):
    from paper_2403_16863_amd import linear
    g = torch.Generator().manual_seed(M + K)

    def values(*shape, sigma=1.0):
        return (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()
    x, w, dy, pre = values(M, K), values(K, N, sigma=K ** -0.5), values(M, N), values(M, N)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    linear.gemm_linear_bwd(dy, x, w, pre, dx, dw, None, kind)
    dz = act_grad(pre.double(), kind, dy.double())
    rounded = dz.to(dtype).double()
    # The kernel's own dz is within 2^-18 of |dy| of this one (the exponential's argument, 20 at most where it counts, is a few roundings off in 32 bits, and
    # the slopes change by 1.2 at most for a unit of it): where that is a border between two numbers, it may have been rounded to the other.
    own = 2.0 ** -18 * dy.double().abs() * (kind != "relu")
    other = ((dz + own).to(dtype).double() - (dz - own).to(dtype).double()).abs()
    x64, w64 = x.double(), w.double()
    for name, got, product, size, border, exact, n in (
            ("dx", dx, rounded @ w64.t(), rounded.abs() @ w64.abs().t(), other @ w64.abs().t(), dz @ w64.t(), N),
            ("dw", dw, x64.t() @ rounded, x64.abs().t() @ rounded.abs(), x64.abs().t() @ other, x64.t() @ dz, M)):
        bound = U[dtype] * product.abs() + TINY[dtype] + (n + 8) * 2.0 ** -24 * size + border
        worst = ((got.double() - product).abs() / bound).max().item()
        assert worst <= 1, f"{name}: {worst:.3g} of the bound"
        # Against dz unrounded: two roundings that know nothing of each other, each 3^-1/2 of half a step in the mean square (half a step: at most U of
        # the value), and a twentieth for what the mean of so many is off by
        off = ((got.double() - exact).norm() / exact.norm()).item()
        assert off <= 1.05 * (2 / 3) ** 0.5 * U[dtype], name
