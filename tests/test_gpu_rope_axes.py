"""Norms with a rotation by positions on several axes, forward and backward, against the formulas in 64 bits (tests/kv4_ref.py)."""
import numpy as np
import pytest
import torch

from tests import kv4_ref as R
from tests.block_ref import same
from tests.test_gpu_kv4 import DTYPES, U, f64, tables_for

pytestmark = pytest.mark.gpu

ROWS = 50


def inputs(B, N, H, Hkv, d, axes, dtype, weights, seed=0):
    g = torch.Generator().manual_seed(seed + N + axes)
    qkv = torch.randn(B, N, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
    dqk = torch.randn(B, N, H + Hkv, d, generator=g).to(dtype).cuda()
    w = [None, None] if weights is None else [(torch.rand(d, generator=g) + 0.5).to(weights).cuda() for _ in range(2)]
    positions = torch.randint(0, ROWS, (B, N, axes), generator=g).int().cuda()
    c, s = tables_for(d, ROWS)
    return qkv[:, :, :H], qkv[:, :, H:H + Hkv], dqk[:, :, :H], dqk[:, :, H:], w, c, s, positions


def angles(c, s, positions, axes):
    """Each pair's cosine and sine, [B,N,1,d/2], from its own axis's row."""
    c, s, at = f64(c), f64(s), positions.cpu().numpy()
    co, si = np.ones((*at.shape[:2], 1, len(axes))), np.zeros((*at.shape[:2], 1, len(axes)))
    for p, a in enumerate(axes):
        if a != 255:
            co[:, :, 0, p], si[:, :, 0, p] = c[at[:, :, a], p], s[at[:, :, a], p]
    return co, si


# sections of pairs (d / 2 in all at most), in one run each or in turns: borders on and off multiples of 8, empty ones, pairs that are not turned, four axes
AXES = [(128, (16, 24, 24), False), (128, (21, 22, 21), False), (128, (24, 20, 20), True), (64, (4, 14, 14), False), (64, (32,), False), (64, (0, 8, 16), False),
        (128, (1, 2, 3, 5), False), (64, (9, 3, 11, 7), True), (128, (0, 0), False)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("weights", [None, "own", torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,sections,alternating", AXES)
def test_forward_and_backward_match_the_formulas(d, sections, alternating, interleaved, weights, dtype):
    from paper_2403_16863_amd import rope
    weights = dtype if weights == "own" else weights
    eps, axes = 1e-5, rope.axes_of_pairs(sections, d, alternating)
    for B, N, H, Hkv in ((1, 1, 3, 1), (2, 37, 12, 4)):
        q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, len(sections), dtype, weights)
        qo = torch.full((B, H, N, d), float("nan"), dtype=dtype, device="cuda").transpose(1, 2)
        ko = torch.full((B, N, Hkv, d), float("nan"), dtype=dtype, device="cuda")
        rope.qk_norm_rope_axes(q, k, qo, ko, c, s, positions, axes, qw, kw, eps, interleaved)
        dq, dk = torch.full_like(qo, float("nan")), torch.full((B, Hkv, N, d), float("nan"), dtype=dtype, device="cuda").transpose(1, 2)
        dqw, dkw = ((torch.full((d,), float("nan"), device="cuda") for _ in range(2)) if weights else (None, None))
        rope.qk_norm_rope_axes_bwd(dqo, dko, q if weights else None, k if weights else None, dq, dk, c, s, positions, axes, qw, kw, dqw, dkw, eps,
                                   interleaved)
        co, si = angles(c, s, positions, axes)
        for x, w, y, dy, dx, dw in ((q, qw, qo, dqo, dq, dqw), (k, kw, ko, dko, dk, dkw)):
            w64 = None if w is None else f64(w)
            want = R.norm_rope(f64(x), w64, co, si, eps, interleaved)
            # half a step of the result's type, and about 8 roundings in 32 bits of the pair's two terms
            terms = np.sqrt((want ** 2).sum(-1, keepdims=True))
            assert (np.abs(f64(y) - want) <= U[dtype] * np.abs(want) + 2.0 ** -20 * terms).all()
            gx, gw = R.norm_rope_bwd(f64(dy), f64(x), w64, co, si, eps, interleaved)
            size = np.abs(gx).max(-1, keepdims=True) + np.abs(f64(dy)).max(-1, keepdims=True)
            assert (np.abs(f64(dx) - gx) <= U[dtype] * np.abs(gx) + 2.0 ** -18 * size * (1 + (0 if w is None else np.abs(f64(x)).max()))).all()
            if w is not None:
                n = B * N * x.shape[2]
                bound = 2.0 ** -24 * (8 + n) * np.abs(f64(dy)).max() * np.abs(f64(x)).max() * 4 * n ** 0.5 + 1e-6
                assert (np.abs(f64(dw) - gw) <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_equal_positions_are_the_rotation_by_one(d, dtype):
    """With the same position on every axis the result is qk_norm_rope's, and so is one axis.  Not bit for bit: of the two products of a pair's channel, a c - b s,
    one is fused with the sum, and which is each kernel's own compilation's choice, so that the sums in 32 bits may differ by 2^-24 (|a c| + |b s|) and a rounding of
    their own, below 2^-22 (|a| + |b|), and their roundings to 16 bits by a step then."""
    from paper_2403_16863_amd import rope
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(2, 33, 4, 2, d, 1, dtype, dtype)
    one = [torch.empty(2, 33, n, d, dtype=dtype, device="cuda") for n in (4, 2, 4, 2)]
    weights = [torch.empty(d, device="cuda") for _ in range(4)]
    at = positions[..., 0].contiguous()
    rope.qk_norm_rope(q, k, one[0], one[1], c, s, at, qw, kw)
    rope.qk_norm_rope_bwd(dqo, dko, q, k, one[2], one[3], c, s, at, qw, kw, *weights[:2])
    for p, sections, alternating in ((positions, (d // 2,), False), (positions.expand(2, 33, 3).contiguous(), (5, 7, d // 2 - 12), False),
                                     (positions.expand(2, 33, 2).contiguous(), (d // 4, d // 4), True)):
        axes = rope.axes_of_pairs(sections, d, alternating)
        two = [torch.empty_like(t) for t in one]
        rope.qk_norm_rope_axes(q, k, two[0], two[1], c, s, p, axes, qw, kw)
        rope.qk_norm_rope_axes_bwd(dqo, dko, q, k, two[2], two[3], c, s, p, axes, qw, kw, *weights[2:])
        for a, b in zip(one, two):
            size = a.float().abs().amax(-1, keepdim=True)              # a pair's channels are d/2 apart: the token's largest bounds both
            assert ((a.float() - b.float()).abs() <= 2 * U[dtype] * a.float().abs() + 2.0 ** -19 * size).all()
        for a, b, x, dy in ((weights[0], weights[2], q, dqo), (weights[1], weights[3], k, dko)):
            # terms g n with |g| <= 2 |dy| and |n| <= |x| / rms(x), each g off by 2^-22 of its pair
            n = x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True))
            assert ((a - b).abs() <= 2.0 ** -20 * 2 * dy.float().abs().max() * n.abs().sum((0, 1, 2)).max()).all()


def test_positions_outside_the_table_touch_their_own_pairs():
    from paper_2403_16863_amd import rope
    d, dtype = 64, torch.float16
    q, _, dqo, _, (qw, _), c, s, positions = inputs(2, 9, 3, 1, d, 3, dtype, dtype)
    axes = rope.axes_of_pairs((8, 10, 6), d)
    want, got = torch.empty(2, 9, 3, d, dtype=dtype, device="cuda"), torch.empty(2, 9, 3, d, dtype=dtype, device="cuda")
    rope.qk_norm_rope_axes(q, None, want, None, c, s, positions, axes, qw)
    positions[0, 4, 1], positions[1, 8, 2] = ROWS, -1
    rope.qk_norm_rope_axes(q, None, got, None, c, s, positions, axes, qw)
    bad = torch.zeros(2, 9, 3, d, dtype=torch.bool, device="cuda")
    for p in range(d // 2):
        for ch in (p, p + d // 2):
            bad[0, 4, :, ch] |= axes[p] == 1
            bad[1, 8, :, ch] |= axes[p] == 2
    assert torch.isnan(got[bad]).all() and same(got[~bad], want[~bad])
    dq, dw = torch.empty_like(want), torch.empty(d, device="cuda")
    rope.qk_norm_rope_axes_bwd(dqo, None, q, None, dq, None, c, s, positions, axes, qw, None, dw, None)
    assert torch.isnan(dq[0, 4]).all() and torch.isnan(dq[1, 8]).all() and not torch.isnan(dq[0, :4]).any() and not torch.isnan(dq[1, :8]).any()
    rope.qk_norm_rope_axes_bwd(dqo, None, None, None, dq, None, c, s, positions, axes)       # without a weight pairs do not meet
    assert torch.isnan(dq[bad]).all() and not torch.isnan(dq[~bad]).any()


def test_the_same_every_time_on_streams_from_graphs_and_in_python():
    from paper_2403_16863_amd import rope
    B, N, H, Hkv, d = 2, 600, 8, 2, 128
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, 3, torch.bfloat16, torch.bfloat16)
    axes = rope.axes_of_pairs((20, 22, 22), d)

    def fresh():
        return [torch.full((B, N, n, d), float("nan"), dtype=torch.bfloat16, device="cuda") for n in (H, Hkv, H, Hkv)] + \
            [torch.full((d,), float("nan"), device="cuda") for _ in range(2)]

    def call(o, **more):
        rope.qk_norm_rope_axes(q, k, o[0], o[1], c, s, positions, axes, qw, kw, stream=more.get("stream"))
        rope.qk_norm_rope_axes_bwd(dqo, dko, q, k, o[2], o[3], c, s, positions, axes, qw, kw, o[4], o[5], **more)
        return o
    want = call(fresh())
    assert all(same(a, b) for a, b in zip(call(fresh()), want))
    space = torch.empty(rope.qk_norm_rope_bwd_workspace(B, N, H, Hkv, d), dtype=torch.uint8, device="cuda")
    assert all(same(a, b) for a, b in zip(call(fresh(), workspace=space), want))             # the Python path
    side, outs = torch.cuda.Stream(), fresh()
    with pytest.raises(ValueError, match="workspace"):
        call(fresh(), stream=side.cuda_stream)
    torch.cuda.synchronize()
    call(outs, stream=side.cuda_stream, workspace=space)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs)
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(outs, want)) and all(same(a, b) for a, b in zip(call(fresh()), want))
