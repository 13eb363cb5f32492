"""The rotation by several axes where a workgroup goes through several tiles of tokens, and held to one axis's more closely than elsewhere."""
import pytest
import torch

from tests.block_ref import DTYPES, TINY, U, same
from tests.test_gpu_rope_axes import ROWS, angles, inputs

pytestmark = pytest.mark.gpu


def turn(a, co, si, interleaved):
    m, n = (a[..., 0::2], a[..., 1::2]) if interleaved else a.chunk(2, -1)
    p, q = m * co - n * si, n * co + m * si
    return torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved,weights", [(False, True), (True, True), (False, False)])
@pytest.mark.parametrize("B,N,H,Hkv,d,sections,alternating", [(2, 8317, 2, 1, 64, (4, 14, 14), False), (3, 5639, 3, 2, 128, (20, 22, 20), True)])
def test_many_tiles_of_tokens(B, N, H, Hkv, d, sections, alternating, interleaved, weights, dtype):
    """More tiles of 8 tokens than a backward pass has workgroups (2048 at most): each goes through several, and adds the weights' gradients over them."""
    from paper_2403_16863_amd import rope
    assert B * N > 8 * 2048 and N % 8
    eps, axes = 1e-5, rope.axes_of_pairs(sections, d, alternating)
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, len(sections), dtype, dtype if weights else None)
    out = [torch.full((B, N, n, d), float("nan"), dtype=dtype, device="cuda") for n in (H, Hkv, H, Hkv)]
    grads = [torch.full((d,), float("nan"), device="cuda") if weights else None for _ in range(2)]
    rope.qk_norm_rope_axes(q, k, out[0], out[1], c, s, positions, axes, qw, kw, eps, interleaved)
    rope.qk_norm_rope_axes_bwd(dqo, dko, q if weights else None, k if weights else None, out[2], out[3], c, s, positions, axes, qw, kw, *grads, eps, interleaved)
    co, si = (torch.from_numpy(t).cuda() for t in angles(c, s, positions, axes))
    for x, w, y, dy, dx, dw in ((q, qw, out[0], dqo, out[2], grads[0]), (k, kw, out[1], dko, out[3], grads[1])):
        x, dy, w = x.double(), dy.double(), None if w is None else w.double()
        r = 1 if w is None else (x.square().mean(-1, keepdim=True) + eps).rsqrt()
        n = x * r
        want = turn(n if w is None else n * w, co, si, interleaved)
        # half a step of the result's type, and a few roundings in 32 bits of the pair's two terms, which the head's length bounds
        close(y, want, U[dtype] * want.abs() + TINY[dtype] + 2.0 ** -20 * want.norm(dim=-1, keepdim=True), "out")
        g = turn(dy, co, -si, interleaved)
        size = dy.norm(dim=-1, keepdim=True)                           # bounds each channel of g
        if w is None:
            close(dx, g, U[dtype] * g.abs() + TINY[dtype] + 2.0 ** -20 * size, "dx")
            continue
        p = g * w
        want = r * (p - n * (p * n).mean(-1, keepdim=True))
        # the second term has a mean of d products, at most d^-1/2 of the lengths of p and n each; n is d^1/2 long
        each = r * w.max() * size * (1 + n.abs())
        close(dx, want, U[dtype] * want.abs() + TINY[dtype] + 2.0 ** -19 * each, "dx")
        # a sum of as many terms in 32 bits, each off by 2^-20 of what bounds it
        terms = x.shape[0] * x.shape[1] * x.shape[2]
        close(dw, (g * n).sum((0, 1, 2)), (terms + 8) * 2.0 ** -24 * (g * n).abs().sum((0, 1, 2)) + 2.0 ** -20 * (size * n.abs()).sum((0, 1, 2)), "dw")


def close(got, want, bound, what):
    error = (got.double() - want).abs()
    assert torch.isfinite(error).all(), what
    worst = (error / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_equal_positions_are_within_a_fused_product_of_one_axis(d, interleaved, dtype):
    """A pair's result by several axes at one position beside qk_norm_rope's: one of its two products may be fused with the sum in one kernel and the other
    in the other, so the sums in 32 bits differ by 2^-24 of each product and of the sum at most, below 2^-22 of the pair's length together; then each is rounded, to the
    same number or a neighbour.  (Held for each pair by its own two channels.)"""
    from paper_2403_16863_amd import rope
    B, N = 2, 65
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, 4, 2, d, 1, dtype, dtype)
    at = positions[..., 0].contiguous()
    one = [torch.empty(B, N, n, d, dtype=dtype, device="cuda") for n in (4, 2, 4, 2)]
    rope.qk_norm_rope(q, k, one[0], one[1], c, s, at, qw, kw, interleaved=interleaved)
    rope.qk_norm_rope_bwd(dqo, dko, None, None, one[2], one[3], c, s, at, interleaved=interleaved)
    for sections, alternating in (((d // 2,), False), ((5, 7, d // 2 - 12), False), ((d // 4, d // 4), True)):
        axes, p = rope.axes_of_pairs(sections, d, alternating), positions.expand(B, N, len(sections)).contiguous()
        two = [torch.empty_like(t) for t in one]
        rope.qk_norm_rope_axes(q, k, two[0], two[1], c, s, p, axes, qw, kw, interleaved=interleaved)
        rope.qk_norm_rope_axes_bwd(dqo, dko, None, None, two[2], two[3], c, s, p, axes, interleaved=interleaved)
        for a, b in zip(one, two):
            a, b = a.double(), b.double()
            m, n = (a[..., 0::2], a[..., 1::2]) if interleaved else a.chunk(2, -1)
            length = (m.square() + n.square()).sqrt() * (1 + 2 * U[dtype])             # of the rounded pair
            length = torch.stack((length, length), -1).flatten(-2) if interleaved else torch.cat((length, length), -1)
            assert ((a - b).abs() <= 2 * U[dtype] * torch.maximum(a.abs(), b.abs()) + 2 * TINY[dtype] + 2.0 ** -22 * length).all()
            assert (a == b).double().mean() > 0.99                     # (neighbours only where a border between two numbers is as near as that)


def test_all_rows_of_the_table_in_one_call():
    """Every position of the table on every axis, forward and back: a rotation and its inverse, which only the two roundings keep from the input."""
    from paper_2403_16863_amd import rope
    d, dtype = 64, torch.float16
    q, _, _, _, _, c, s, _ = inputs(1, ROWS, 1, 1, d, 2, dtype, None)
    n = torch.arange(ROWS, device="cuda")
    positions = torch.stack((n, ROWS - 1 - n), -1).int()[None].contiguous()
    axes, there, back = rope.axes_of_pairs((9, 23), d), torch.empty(1, ROWS, 1, d, dtype=dtype, device="cuda"), torch.empty(1, ROWS, 1, d, dtype=dtype, device="cuda")
    rope.qk_norm_rope_axes(q, None, there, None, c, s, positions, axes)
    rope.qk_norm_rope_axes_bwd(there, None, None, None, back, None, c, s, positions, axes)
    m, k = q.double().chunk(2, -1)
    length = (m.square() + k.square()).sqrt().repeat(1, 1, 1, 2)
    # half a step of each of the pair's two turned channels, at most 2^1/2 of the pair's, and half a step of the result; the table's own c^2 + s^2 and the sums in 32 bits
    assert ((back.double() - q.double()).abs() <= U[dtype] * (2 ** 0.5 * length + q.double().abs()) * 1.001 + 2.0 ** -20 * length + 2 * TINY[dtype]).all()
    assert not same(there, q)
