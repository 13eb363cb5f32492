"""The norms with the residual stream where a workgroup goes through several rounds of tokens or several sequences."""
import pytest
import torch

from tests.block_ref import same

pytestmark = pytest.mark.gpu


def test_as_many_sequences_as_a_call_takes():
    """2^31 - 1 sequences of a token, each with its own gate: dh = dy gate in every one of them, the last workgroups' last among them."""
    from paper_2403_16863_amd import norm
    B, C, dtype = 2 ** 31 - 1, 8, torch.bfloat16
    if torch.cuda.mem_get_info()[0] < 2 * 2 * B * C + (8 << 30):
        pytest.skip("needs 77 GB")
    g = torch.Generator().manual_seed(14)
    dy, h = (torch.randn(1, 1, C, generator=g).to(dtype).cuda() for _ in range(2))
    part, rows = 1 << 28, torch.randn(1 << 20, C, generator=g).to(dtype).cuda()
    gate, dh = torch.empty(B, C, dtype=dtype, device="cuda"), torch.full((B, 1, C), float("nan"), dtype=dtype, device="cuda")
    for i in range(0, B, 1 << 20):
        gate[i:i + (1 << 20)] = rows[:min(1 << 20, B - i)]
    norm.residual_norm_bwd(dy.expand(B, 1, C), None, None, h.expand(B, 1, C), None, dh, gate)
    for i in range(0, B, part):
        assert same(dh[i:i + part, 0], gate[i:i + part] * dy[0])
