"""Norms with rotation, forward and backward, against the formulas in 64 bits (tests/kv4_ref.py) and against differences."""
import numpy as np
import pytest
import torch

from tests import kv4_ref as R
from tests.test_gpu_kv4 import DTYPES, U, f64, tables_for

pytestmark = pytest.mark.gpu


def inputs(B, N, H, Hkv, d, dtype, weights, seed=0):
    g = torch.Generator().manual_seed(seed + N)
    qkv = torch.randn(B, N, H + 2 * Hkv, d, generator=g).to(dtype).cuda()
    dqk = torch.randn(B, N, H + Hkv, d, generator=g).to(dtype).cuda()
    w = [None, None] if weights is None else [(torch.rand(d, generator=g) + 0.5).to(weights).cuda() for _ in range(2)]
    positions = torch.randint(0, 50, (B, N), generator=g).int().cuda()
    c, s = tables_for(d, 50)
    return qkv[:, :, :H], qkv[:, :, H:H + Hkv], dqk[:, :, :H], dqk[:, :, H:], w, c, s, positions


def angles(c, s, positions):
    at = positions.long()
    return f64(c[at][:, :, None]), f64(s[at][:, :, None])


SIZES = [(1, 1, 1, 1, 64), (1, 1, 32, 8, 128), (3, 7, 5, 1, 64), (2, 9, 3, 3, 128), (1, 65, 12, 4, 64), (2, 33, 40, 10, 128)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("weights", [None, "own", torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,N,H,Hkv,d", SIZES)
def test_forward_and_backward_match_the_formulas(B, N, H, Hkv, d, interleaved, weights, dtype):
    from paper_2403_16863_amd import rope
    weights = dtype if weights == "own" else weights
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, dtype, weights)
    eps = 1e-5
    # head-major outputs for the one, token-major for the other
    qo = torch.full((B, H, N, d), float("nan"), dtype=dtype, device="cuda").transpose(1, 2)
    ko = torch.full((B, N, Hkv, d), float("nan"), dtype=dtype, device="cuda")
    rope.qk_norm_rope(q, k, qo, ko, c, s, positions, qw, kw, eps, interleaved)
    dq, dk = torch.full_like(qo, float("nan")), torch.full((B, Hkv, N, d), float("nan"), dtype=dtype, device="cuda").transpose(1, 2)
    dqw, dkw = ((torch.full((d,), float("nan"), device="cuda") for _ in range(2)) if weights else (None, None))
    rope.qk_norm_rope_bwd(dqo, dko, q if weights else None, k if weights else None, dq, dk, c, s, positions, qw, kw, dqw, dkw, eps, interleaved)
    co, si = angles(c, s, positions)
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


def test_gradients_match_differences():
    """Central differences of the 64-bit forward along random directions, at eps of the size of the mean square."""
    from paper_2403_16863_amd import rope
    B, N, H, d, eps = 2, 3, 2, 64, 0.5
    q, _, dqo, _, (qw, _), c, s, positions = inputs(B, N, H, 1, d, torch.float16, torch.float32)
    dq, dqw = torch.empty_like(q), torch.empty(d, device="cuda")
    rope.qk_norm_rope_bwd(dqo, None, q, None, dq, None, c, s, positions, qw, None, dqw, None, eps)
    co, si = angles(c, s, positions)
    rng = np.random.default_rng(0)
    x, w, dy, h = f64(q), f64(qw), f64(dqo), 1e-5
    for _ in range(8):
        vx, vw = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        loss = lambda a: (R.norm_rope(x + a * vx, w + a * vw, co, si, eps, False) * dy).sum()  # noqa: E731
        slope = (loss(h) - loss(-h)) / (2 * h)
        got = (f64(dq) * vx).sum() + (f64(dqw) * vw).sum()
        # each gradient is rounded to binary16 (half a step, random signs: four deviations of the sum)
        tol = 4 * 2.0 ** -11 * np.sqrt(((f64(dq) * vx) ** 2).sum()) + 1e-4
        assert abs(got - slope) <= tol


@pytest.mark.parametrize("d", [64, 128])
def test_one_tensor_in_place_and_positions_outside_the_table(d):
    from paper_2403_16863_amd import rope
    q, k, dqo, _, (qw, _), c, s, positions = inputs(2, 11, 4, 2, d, torch.bfloat16, torch.bfloat16)
    want = torch.empty(2, 11, 4, d, dtype=torch.bfloat16, device="cuda")
    rope.qk_norm_rope(q, None, want, None, c, s, positions, qw)
    mine = q.clone()
    rope.qk_norm_rope(mine, None, mine, None, c, s, positions, qw)
    assert torch.equal(mine.view(torch.int16), want.view(torch.int16))
    alone = torch.empty_like(want)
    rope.qk_norm_rope(None, q, None, alone, c, s, positions, None, qw)     # as keys, without queries
    assert torch.equal(alone.view(torch.int16), want.view(torch.int16))
    both, ko = torch.empty_like(want), torch.empty(2, 11, 2, d, dtype=torch.bfloat16, device="cuda")
    rope.qk_norm_rope(q, k, both, ko, c, s, positions, qw)          # a norm for the queries alone
    assert torch.equal(both.view(torch.int16), want.view(torch.int16))
    co, si = angles(c, s, positions)
    plain = R.rotate(f64(k), co, si, False)
    assert (np.abs(f64(ko) - plain) <= 2.0 ** -8 * np.abs(plain) + 2.0 ** -20 * np.abs(f64(k)).max()).all()
    positions[0, 3], positions[1, 10] = -1, 50
    rope.qk_norm_rope(q, None, both, None, c, s, positions, qw)
    bad = torch.zeros(2, 11, dtype=torch.bool, device="cuda")
    bad[0, 3] = bad[1, 10] = True
    assert torch.isnan(both[bad]).all() and torch.equal(both[~bad].view(torch.int16), want[~bad].view(torch.int16))
    dq, dw = torch.empty_like(want), torch.empty(d, device="cuda")
    rope.qk_norm_rope_bwd(dqo, None, q, None, dq, None, c, s, positions, qw, None, dw, None)
    assert torch.isnan(dq[bad]).all() and not torch.isnan(dq[~bad]).any() and torch.isnan(dw).all()


def test_backward_is_the_same_every_time_on_streams_and_from_graphs():
    from paper_2403_16863_amd import rope
    B, N, H, Hkv, d = 2, 1100, 8, 2, 128
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, torch.bfloat16, torch.bfloat16)

    def call(**more):
        outs = [torch.full((B, N, n, d), float("nan"), dtype=torch.bfloat16, device="cuda") for n in (H, Hkv)]
        outs += [torch.full((d,), float("nan"), device="cuda") for _ in range(2)]
        rope.qk_norm_rope_bwd(dqo, dko, q, k, outs[0], outs[1], c, s, positions, qw, kw, outs[2], outs[3], **more)
        return outs

    def same(a, b):
        return all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, b))
    want = call()
    assert same(call(), want)
    need = rope.qk_norm_rope_bwd_workspace(B, N, H, Hkv, d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with pytest.raises(ValueError, match="workspace"):
        call(stream=side.cuda_stream)
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    outs = [torch.empty((B, N, n, d), dtype=torch.bfloat16, device="cuda") for n in (H, Hkv)] + [torch.empty(d, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    rope.qk_norm_rope_bwd(dqo, dko, q, k, outs[0], outs[1], c, s, positions, qw, kw, outs[2], outs[3], workspace=space, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert same(outs, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rope.qk_norm_rope_bwd(dqo, dko, q, k, outs[0], outs[1], c, s, positions, qw, kw, outs[2], outs[3])
    for _ in range(3):
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same(outs, want)
        assert same(call(), want)


def test_feeds_the_attention_forward():
    """Projections to attn_fwd in its own layout, without a copy between."""
    import paper_2403_16863_amd as A
    from paper_2403_16863_amd import rope
    B, N, H, d = 1, 70, 2, 64
    q, k, _, _, (qw, kw), c, s, positions = inputs(B, N, H, H, d, torch.float16, torch.float16)
    v = torch.randn(B, H, N, d, device="cuda").half()
    qo, ko, out = (torch.empty(B, H, N, d, device="cuda", dtype=torch.float16) for _ in range(3))
    lse = torch.empty(B, H, N, device="cuda")
    rope.qk_norm_rope(q, k, qo.transpose(1, 2), ko.transpose(1, 2), c, s, positions, qw, kw)
    A.attn_fwd(qo, ko, v, out, lse, True, d ** -0.5)
    co, si = angles(c, s, positions)
    q64, k64 = (R.norm_rope(f64(x), f64(w), co, si, 1e-6, False).transpose(0, 2, 1, 3) for x, w in ((q, qw), (k, kw)))
    x = q64 @ k64.transpose(0, 1, 3, 2) * d ** -0.5
    x[..., np.triu(np.ones((N, N), bool), 1)] = -np.inf
    p = np.exp(x - x.max(-1, keepdims=True))
    want = p / p.sum(-1, keepdims=True) @ f64(v)
    # scores from rounded q and k: 2 * 2^-11 * sum |q k| * scale <= 2^-10 * 1.5^2 * 8; probabilities and the result add 2^-11 each
    assert np.abs(f64(out) - want).max() <= (2 * 2.0 ** -10 * 18 + 2 * 2.0 ** -11) * np.abs(f64(v)).max()
