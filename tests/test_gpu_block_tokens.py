"""The operators around the attention for one token and for rows of a prompt, each held to the formulas with the roundings between them followed."""
import pytest
import torch

from tests.block_ref import DTYPES, TINY, U, act, same
from tests.test_gpu_block import weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 9, 33])
def test_hidden_layer_of_tokens_matches_the_formulas(rows, dtype):
    """norm, product with bias and activation, product with bias onto the stream: `hidden` is the kernel's own rounding of its 64-bit value, or a neighbour of it
    where a border between two numbers is within the sums' error, and the result follows from it."""
    from paper_2403_16863_amd import linear, norm
    C, hidden, N = 264, 1032, 33
    w = weights(dtype, C, 2, 2, 64, hidden)
    g = torch.Generator().manual_seed(5)
    x, h = (torch.randn(1, N, C, generator=g).to(dtype).cuda() for _ in range(2))
    whole = torch.empty_like(x), torch.empty_like(x)
    norm.residual_norm(x, h, *whole, None, w["post"], w["norm2"])
    for at in range(0, N, rows):
        part = slice(at, min(N, at + rows))
        n = part.stop - part.start
        y, z = torch.empty_like(x[:, part]), torch.empty_like(x[:, part])
        up, out = torch.empty(n, hidden, dtype=dtype, device="cuda"), torch.empty(n, C, dtype=dtype, device="cuda")
        norm.residual_norm(x[:, part], h[:, part], y, z, None, w["post"], w["norm2"])
        assert same(y, whole[0][:, part]) and same(z, whole[1][:, part])           # a token's sums are its own
        linear.gemm_linear(z[0], w["up"], up, w["up_bias"], activation="silu")
        linear.gemm_linear(up, w["down"], out, w["down_bias"], y[0])
        z64, up64 = z[0].double(), w["up"].double()
        pre = z64 @ up64 + w["up_bias"].double()
        sums = (C + 8) * 2.0 ** -24 * (z64.abs() @ up64.abs() + w["up_bias"].double().abs())
        want = act(pre, "silu")
        off = 1.1 * sums + 2.0 ** -20 * pre.abs()                                  # silu's slope is 1.1 at most; its own error
        border = (want + off).to(dtype).double() - (want - off).to(dtype).double()
        rounded = want.to(dtype).double()
        assert ((up.double() - rounded).abs() <= border).all()
        down = w["down"].double()
        want = rounded @ down + w["down_bias"].double() + y[0].double()
        size = rounded.abs() @ down.abs() + w["down_bias"].double().abs() + y[0].double().abs()
        bound = U[dtype] * want.abs() + TINY[dtype] + (hidden + 8) * 2.0 ** -24 * size + border @ down.abs()
        assert ((out.double() - want).abs() <= bound).all()
        # the bound is small beside what a part left out would change
        assert bound.max() < 0.2 * w["down_bias"].abs().max() and bound.max() < 0.2 * w["up_bias"].abs().max()
