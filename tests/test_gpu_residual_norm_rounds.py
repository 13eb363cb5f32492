"""The norms with the residual stream where a workgroup goes through several rounds of tokens or several sequences."""
import pytest
import torch

from tests import test_gpu_residual_norm as single
from tests.block_ref import DTYPES, same

formulas, FORMS = single.test_forward_and_backward_match_the_formulas, single.FORMS

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


# channels for one to sixteen waves a token, and tokens enough for more than one round of a workgroup both ways: forward from 2048 rounds on, eight waves' tokens
# each.  No number of tokens divides by a round, so that sequences, and with them gates, change inside a workgroup's run.
ROUNDS = [(7, 2401, 72), (9, 1001, 520), (5, 901, 1032), (3, 1411, 1544), (3, 1001, 4096), (3, 701, 4104), (2, 1051, 8200)]


def test_rounds_are_several():
    for B, N, C in ROUNDS:
        waves = next(w for w, most in ((1, 512), (2, 1024), (3, 1536), (4, 2048), (8, 8192), (16, 16384)) if C <= most)
        at_once = max(1, 8 // waves)
        assert -(-B * N // at_once) > 2048 and N % at_once + (at_once == 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate,post,alpha,wide,where", FORMS)
@pytest.mark.parametrize("B,N,C", ROUNDS)
def test_several_rounds_match_the_formulas(B, N, C, gate, post, alpha, wide, where, dtype):
    """Forward and backward, every token and every vector's gradient, as the smaller sizes are tested."""
    formulas(B, N, C, gate, post, alpha, wide, where, dtype)


def test_several_rounds_of_the_stream_in_place():
    """A training size, the stream updated in its own memory, twice from the same beginning and from a graph among eager runs."""
    from paper_2403_16863_amd import norm
    B, N, C, dtype = 2, 1501, 4096, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(15)
    x, h = (torch.randn(B, N, C, generator=g, device="cuda").to(dtype) for _ in range(2))
    gate, post, pre = torch.randn(B, C, generator=g, device="cuda").to(dtype), *(torch.rand(C, generator=g, device="cuda") + 0.5 for _ in range(2))
    y, z, stream, z2 = (torch.empty_like(x) for _ in range(4))
    norm.residual_norm(x, h, y, z, gate, post, pre)

    def run():
        stream.copy_(x)
        norm.residual_norm(stream, h, stream, z2, gate, post, pre)
    run()
    assert same(stream, y) and same(z2, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        stream.fill_(float("nan")), z2.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same(stream, y) and same(z2, z)
        run()
        assert same(stream, y) and same(z2, z)
