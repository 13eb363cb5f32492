"""Pairs of channels without an axis: the rotation by several axes leaves them as they are, whatever their values."""
import pytest
import torch

from tests.block_ref import DTYPES, same
from tests.test_gpu_kv4 import tables_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,sections,alternating", [(64, (8, 10, 6), False), (128, (3, 20, 20), True), (64, (0, 0), False), (128, (1,), False)])
def test_pairs_that_are_not_turned_keep_their_bits(d, sections, alternating, interleaved, dtype):
    """Infinities, NaN and zeros of both signs beside ordinary values, forward and backward."""
    from paper_2403_16863_amd import rope
    B, N, H = 2, 21, 3
    axes = rope.axes_of_pairs(sections, d, alternating)
    g = torch.Generator().manual_seed(d + len(sections))
    c, s = tables_for(d, 50)
    positions = torch.randint(0, 50, (B, N, len(sections)), generator=g).int().cuda()
    x, y, dx = (torch.randn(B, N, H, d, generator=g).to(dtype).cuda() for _ in range(3))
    still = torch.tensor([axes[(ch // 2 if interleaved else ch % (d // 2))] == rope.NO_AXIS for ch in range(d)]).cuda()
    odd = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 1.5, -2.5], dtype=dtype).cuda()
    x[..., still] = odd[torch.randint(0, len(odd), (B, N, H, int(still.sum())), generator=g).cuda()]
    rope.qk_norm_rope_axes(x, None, y, None, c, s, positions, axes, interleaved=interleaved)
    rope.qk_norm_rope_axes_bwd(x, None, None, None, dx, None, c, s, positions, axes, interleaved=interleaved)
    for got in (y, dx):
        a, b = got[..., still], x[..., still]
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and same(torch.where(torch.isnan(b), b, a), b)
        assert torch.isfinite(got[..., ~still]).all()
