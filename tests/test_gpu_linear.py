"""Linear layers' products, forward and backward, against the formulas in 64 bits and against differences."""
import numpy as np
import pytest
import torch

from tests.block_ref import DTYPES, TINY, U, act, act_grad, inside, same

pytestmark = pytest.mark.gpu

KINDS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def values(g, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()


def close(got, want, bound, what=""):
    error = (got.double() - want).abs()
    assert torch.isfinite(error).all(), what
    worst = (error / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


# (tokens, outputs, inputs): single elements to several tiles, sizes on both sides of the tiles' edges, long sums that are split
SIZES = [(1, 8, 8), (1, 264, 4104), (3, 72, 40), (17, 520, 2056), (64, 64, 4096), (130, 136, 200), (257, 264, 72), (100, 1032, 520)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows_of_n", [False, True])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_forward_matches_the_formula(M, N, K, rows_of_n, dtype):
    """All activations, with and without bias, residual and pre, on views inside larger tensors of NaN."""
    from paper_2403_16863_amd import linear
    g = torch.Generator().manual_seed(M + N)
    nan = float("nan")
    x = inside((M, K), dtype, nan)[0].copy_(values(g, (M, K), dtype))
    w = (inside((N, K), dtype, nan)[0].t() if rows_of_n else inside((K, N), dtype, nan, (2, 16))[0]).copy_(values(g, (K, N), dtype, K ** -0.5))
    residual = inside((M, N), dtype, nan)[0].copy_(values(g, (M, N), dtype))
    z0, size0 = x.double() @ w.double(), x.double().abs() @ w.double().abs()
    for i, kind in enumerate(KINDS):
        bias = [None, values(g, (N,), dtype), values(g, (N,), torch.float32)][i % 3]
        res, with_pre = residual if i % 2 else None, i != 1
        out, whole = inside((M, N), dtype, nan, (3, 24))
        pre = inside((M, N), dtype, nan)[0] if with_pre else None
        linear.gemm_linear(x, w, out, bias, res, pre, kind)
        z, size = (z0, size0) if bias is None else (z0 + bias.double(), size0 + bias.double().abs())
        want = act(z, kind) + (0 if res is None else res.double())
        # half a step of the result; K products and a few terms added in 32 bits, under activations of slope 1.13 at most, whose own
        # error is 2^-17 of |z| (a polynomial good to 2^-18.9 and an exponential whose argument is rounded)
        sums = (K + 8) * 2.0 ** -24 * size
        close(out, want, U[dtype] * want.abs() + TINY[dtype] + 1.2 * sums + 2.0 ** -17 * z.abs() + 2.0 ** -23 * want.abs(), (kind, "out"))
        if pre is not None:
            close(pre, z, U[dtype] * z.abs() + TINY[dtype] + sums, (kind, "pre"))
        assert torch.isnan(whole[M:]).all() and torch.isnan(whole[:, N:]).all()     # nothing but the rows is written


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows_of_n,dw_rows_of_n", [(False, False), (True, True), (False, True)])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_backward_matches_the_formulas(M, N, K, rows_of_n, dw_rows_of_n, dtype):
    from paper_2403_16863_amd import linear
    g = torch.Generator().manual_seed(M + 3 * N)
    nan = float("nan")
    x = inside((M, K), dtype, nan)[0].copy_(values(g, (M, K), dtype))
    dy = inside((M, N), dtype, nan)[0].copy_(values(g, (M, N), dtype))
    w = (inside((N, K), dtype, nan)[0].t() if rows_of_n else inside((K, N), dtype, nan)[0]).copy_(values(g, (K, N), dtype))
    for kind in KINDS:
        pre = inside((M, N), dtype, nan)[0].copy_(values(g, (M, N), dtype, 2.0)) if kind != "none" else None
        dx, whole_x = inside((M, K), dtype, nan)
        dw, whole_w = inside((N, K) if dw_rows_of_n else (K, N), dtype, nan)
        dbias = torch.full((N,), nan, device="cuda")
        linear.gemm_linear_bwd(dy, x, w, pre, dx, dw.t() if dw_rows_of_n else dw, dbias, kind)
        dz = dy.double() if kind == "none" else act_grad(pre.double(), kind, dy.double())
        # dz: the slope's own error in 32 bits (2^-15), and its rounding, both of |dy| 1.13 at most
        own = 2.0 ** -15 * dy.double().abs() if kind != "none" else torch.zeros_like(dz)
        each = own + (U[dtype] * dz.abs() + TINY[dtype] if kind != "none" else 0)
        for name, got, want, size, error, n in (("dx", dx, dz @ w.double().t(), dz.abs() @ w.double().abs().t(), each @ w.double().abs().t(), N),
                                                ("dw", dw.t() if dw_rows_of_n else dw, x.double().t() @ dz, x.double().abs().t() @ dz.abs(),
                                                 x.double().abs().t() @ each, M)):
            close(got, want, U[dtype] * want.abs() + TINY[dtype] + (n + 8) * 2.0 ** -24 * size + error, (kind, name))
        close(dbias, dz.sum(0), (M + 8) * 2.0 ** -24 * dz.abs().sum(0) + own.sum(0) + 1e-30, (kind, "dbias"))
        assert torch.isnan(whole_x[M:]).all() and torch.isnan(whole_x[:, K:]).all()
        assert torch.isnan(whole_w[dw.shape[0]:]).all() and torch.isnan(whole_w[:, dw.shape[1]:]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tile", range(16))
def test_every_tile_in_every_layout_and_in_ranges(tile, dtype):
    from paper_2403_16863_amd import linear
    if tile >= linear.linear_num_tiles():
        return
    g = torch.Generator().manual_seed(tile)
    for layout in (linear.ROWS, linear.ROWS_N, linear.TOKENS):
        for M, N, K in ((8, 8, 8), (264, 72, 264), (200, 520, 1096), (72, 264, 2600)):
            k = K - 5 if layout == linear.TOKENS else K                # the tokens are any number
            m = M if layout == linear.TOKENS else M - 3
            a, b = values(g, (m, k), dtype), values(g, (k, N), dtype)
            want, size = a.double() @ b.double(), a.double().abs() @ b.double().abs()
            a, b = a.t().contiguous() if layout == linear.TOKENS else a, b.t().contiguous() if layout == linear.ROWS_N else b
            for ranges in (1, 2, 7):
                c, whole = inside((m, N), dtype, float("nan"))
                space = torch.full((ranges * m * N * 4 + 64,), 255, dtype=torch.uint8, device="cuda")    # NaN
                linear.linear_product(a, b, layout, c, tile, ranges, space)
                close(c, want, U[dtype] * want.abs() + TINY[dtype] + (k + 8) * 2.0 ** -24 * size, (layout, m, N, k, ranges))
                assert torch.isnan(whole[m:]).all() and torch.isnan(whole[:, N:]).all() and (space[ranges * m * N * 4:] == 255).all()


def test_choices_are_within_the_library():
    from paper_2403_16863_amd import linear
    for layout in range(3):
        for M in (8, 64, 4096, 1 << 20):
            for N in (8, 64, 4096):
                for K in (8, 512, 16384):
                    tile, ranges = linear.linear_choice(M, N, K, layout)
                    assert 0 <= tile < linear.linear_num_tiles() and 1 <= ranges <= 32


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_match_differences(kind):
    """Central differences of the 64-bit forward along random directions."""
    from paper_2403_16863_amd import linear
    M, N, K, dtype = 5, 24, 16, torch.float16
    g = torch.Generator().manual_seed(1)
    x, w, dy, bias = values(g, (M, K), dtype), values(g, (K, N), dtype, 0.4), values(g, (M, N), dtype), values(g, (N,), torch.float32)
    out, pre, dx, dw, dbias = (torch.empty(s, dtype=t, device="cuda") for s, t in (((M, N), dtype), ((M, N), dtype), ((M, K), dtype), ((K, N), dtype),
                                                                                  ((N,), torch.float32)))
    linear.gemm_linear(x, w, out, bias, None, pre, kind)
    linear.gemm_linear_bwd(dy, x, w, pre, dx, dw, dbias, kind)
    rng = np.random.default_rng(0)
    for _ in range(8):
        vx, vw, vb = (torch.from_numpy(rng.standard_normal(s)).cuda() for s in ((M, K), (K, N), (N,)))
        h = 1e-6

        def loss(a):
            return (act((x.double() + a * vx) @ (w.double() + a * vw) + bias.double() + a * vb, kind) * dy.double()).sum().item()
        slope = (loss(h) - loss(-h)) / (2 * h)
        got = ((dx.double() * vx).sum() + (dw.double() * vw).sum() + (dbias.double() * vb).sum()).item()
        # dx, dw and dz are rounded to binary16, and pre, at which the slope is taken (slopes change by 1.2 at most for each unit): four
        # deviations of the sums of those errors; a relu's pre within its rounding of 0 does not occur here
        z = (x.double() @ w.double() + bias.double())
        through = (vx @ w.double() + x.double() @ vw)
        parts = [dx.double() * vx, dw.double() * vw, dy.double() * through * 1.13, 1.2 * dy.double() * z * (through + vb)]
        assert abs(got - slope) <= 4 * 2.0 ** -11 * sum((p ** 2).sum().item() for p in parts) ** 0.5 + 1e-4


@pytest.mark.parametrize("kind", KINDS)
def test_values_at_the_ends_of_the_activations(kind):
    """Large arguments, infinities and NaN, in the forward's order and no other: rows do not meet."""
    from paper_2403_16863_amd import linear
    N, dtype = 8, torch.bfloat16
    z = torch.tensor([0.0, -0.0, 1e-3, -1e-3, 5.0, -5.0, -9.0, 20.0, -20.0, 80.0, -80.0, 200.0, -200.0, 3e38, -3e38, float("inf"), float("nan")], device="cuda")
    x = torch.zeros(len(z), 8, device="cuda", dtype=dtype)
    x[:, 0] = z.to(dtype)
    w = torch.zeros(8, N, device="cuda", dtype=dtype)
    w[0] = 1
    w[1:] = 0
    out = torch.empty(len(z), N, device="cuda", dtype=dtype)
    linear.gemm_linear(x, w, out, activation=kind)
    want = act(x[:, :1].double(), kind).expand(-1, N)
    finite = torch.isfinite(want)
    # 32 bits flush what lies below 2^-126, and the gelu's cube ends at 7e12, where the form has been z or 0 for long
    assert (torch.where(finite, (out.double() - want).abs(), 0.0) <= torch.where(finite, 2.0 ** -8 * want.abs() * 1.01 + 1e-37, 0.0)).all()
    assert (torch.isnan(out) == torch.isnan(want)).all() and (out[-2] == float("inf")).all()
    # the slopes: 0 and 1 far out
    dx, dy = torch.empty_like(x), torch.ones_like(out)
    pre = x[:, :1].expand(-1, N).contiguous()
    dbias = torch.empty(N, device="cuda")
    linear.gemm_linear_bwd(dy, x, w, pre, dx, None, dbias, kind)
    far = act_grad(x[:, 0].double(), kind, torch.ones(len(z), device="cuda", dtype=torch.float64))
    far[-2] = 1                                                         # (the limit; the formulas have infinity times 0 there)
    got = dx[:, 0].double() / N                                         # (w's row 0 is 1: dx sums N equal terms)
    assert ((got - far).abs()[:-1] <= 2.0 ** -7 * far.abs()[:-1] + 2.0 ** -15).all() and (kind == "none" or torch.isnan(got[-1]))
    pre[-2] = -float("inf")
    linear.gemm_linear_bwd(dy, x, w, pre, dx, None, dbias, kind)
    assert (dx[-2, 0] == (N if kind == "none" else 0)).all()


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    from paper_2403_16863_amd import linear
    M, N, K, dtype = 70, 72, 520, torch.float16
    g = torch.Generator().manual_seed(2)
    x, w = values(g, (M, K), dtype), values(g, (K, N), dtype)
    want = torch.empty(M, N, device="cuda", dtype=dtype)
    linear.gemm_linear(x, w, want)
    bad_x, bad_w = x.clone(), w.clone()
    bad_x[33, 519], bad_w[519, 41] = float("nan"), float("inf")
    out = torch.empty_like(want)
    linear.gemm_linear(bad_x, bad_w, out)
    assert torch.isnan(out[33]).all() and not torch.isfinite(out[:, 41]).any()
    keep = torch.ones(M, N, dtype=torch.bool, device="cuda")
    keep[33], keep[:, 41] = False, False
    assert same(out[keep], want[keep])


def test_in_place_residual_joint_buffers_and_the_python_path():
    """The stream updated in place, out among the columns of the tensor that x and the residual lie in, and the path of calls that are not plain."""
    from paper_2403_16863_amd import linear
    M, N, K, dtype = 150, 72, 264, torch.bfloat16
    g = torch.Generator().manual_seed(3)
    x, w, r, bias = values(g, (M, K), dtype), values(g, (K, N), dtype, 0.1), values(g, (M, N), dtype), values(g, (N,), dtype)
    want, pre = torch.empty(M, N, device="cuda", dtype=dtype), torch.empty(M, N, device="cuda", dtype=dtype)
    linear.gemm_linear(x, w, want, bias, r, pre, "silu")
    mine = r.clone()
    linear.gemm_linear(x, w, mine, bias, mine, None, "silu")
    assert same(mine, want)
    joint = torch.cat((x, r, torch.zeros_like(r)), 1)
    linear.gemm_linear(joint[:, :K], w, joint[:, K + N:], bias, joint[:, K:K + N], None, "silu")
    assert same(joint[:, K + N:], want) and same(joint[:, :K], x) and same(joint[:, K:K + N], r)
    other = torch.empty_like(want)
    linear.gemm_linear(x, w, other, bias, r, None, "silu", workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert same(other, want)
    dy = values(g, (M, N), dtype)
    outs = [[torch.empty(s, dtype=t, device="cuda") for s, t in (((M, K), dtype), ((K, N), dtype), ((N,), torch.float32))] for _ in range(2)]
    linear.gemm_linear_bwd(dy, x, w, pre, *outs[0], "silu")
    space = torch.empty(linear.gemm_linear_bwd_workspace(M, N, K, "silu"), dtype=torch.uint8, device="cuda")
    linear.gemm_linear_bwd(dy, x, w, pre, *outs[1], "silu", workspace=space)
    assert all(same(a, b) for a, b in zip(*outs))
    # one gradient alone is the same as among the others
    for i in range(3):
        alone = [None] * 3
        alone[i] = torch.empty_like(outs[0][i])
        linear.gemm_linear_bwd(dy, x if i == 1 else None, w if i == 0 else None, pre, *alone, "silu")
        assert same(alone[i], outs[0][i])


def test_the_same_every_time_on_streams_and_from_graphs():
    """Sizes that split the sums: with torch's memory, on another stream with and without a workspace, and replayed among eager work."""
    from paper_2403_16863_amd import linear
    M, N, K, dtype = 24, 264, 8200, torch.bfloat16
    g = torch.Generator().manual_seed(4)
    x, w, dy, pre = values(g, (M, K), dtype), values(g, (K, N), dtype, 0.01), values(g, (M, N), dtype), values(g, (M, N), dtype)
    assert linear.gemm_linear_workspace(M, N, K) > 0

    def fresh():
        return [torch.full(s, float("nan"), dtype=t, device="cuda") for s, t in (((M, N), dtype), ((M, K), dtype), ((K, N), dtype), ((N,), torch.float32))]

    def call(outs, stream=None, spaces=(None, None)):
        linear.gemm_linear(x, w, outs[0], activation="gelu", workspace=spaces[0], stream=stream)
        linear.gemm_linear_bwd(dy, x, w, pre, *outs[1:], "gelu", workspace=spaces[1], stream=stream)
        return outs
    want = call(fresh())
    assert all(same(a, b) for a, b in zip(call(fresh()), want))
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="workspace"):
        linear.gemm_linear_bwd(dy, x, w, pre, *fresh()[1:], "gelu", stream=side.cuda_stream)
    spaces = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (linear.gemm_linear_workspace(M, N, K),
                                                                         linear.gemm_linear_bwd_workspace(M, N, K, "gelu"))]
    outs = fresh()
    torch.cuda.synchronize()
    call(outs, side.cuda_stream, spaces)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, want))
    whole = fresh()[0]
    torch.cuda.synchronize()
    linear.gemm_linear(x, w, whole, activation="gelu", stream=side.cuda_stream)        # no memory: the sums are not split
    torch.cuda.synchronize()
    z = x.double() @ w.double()
    close(whole, act(z, "gelu"), 2.0 ** -8 * act(z, "gelu").abs() + 2.0 ** -17 * z.abs() + 2 * K * 2.0 ** -24 * (x.double().abs() @ w.double().abs()))
    graphs, outs = [], [fresh(), fresh()]
    for o in outs:                                                      # two graphs, each with memory of its own
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(o)
    for _ in range(3):
        for o in outs:
            for t in o:
                t.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for o in outs for a, b in zip(o, want))
        assert all(same(a, b) for a, b in zip(call(fresh()), want))


def test_rows_far_behind_32_bits():
    """A wide stride: rows beyond 2^32 bytes of their matrix's start."""
    from paper_2403_16863_amd import linear
    M, N, K, dtype = 1100, 64, 64, torch.float16
    stride = 1 << 21
    if torch.cuda.mem_get_info()[0] < 3 * 2 * M * stride:
        pytest.skip("needs 14 GB")
    x = torch.empty(M * stride, dtype=dtype, device="cuda").view(M, stride)[:, :K]
    out = torch.empty(M * stride, dtype=dtype, device="cuda").view(M, stride)[:, 64:64 + N]
    g = torch.Generator().manual_seed(5)
    x.copy_(values(g, (M, K), dtype))
    w, dense = values(g, (K, N), dtype), torch.empty(M, N, dtype=dtype, device="cuda")
    linear.gemm_linear(x, w, out, activation="relu")
    linear.gemm_linear(x.contiguous(), w, dense, activation="relu")
    assert same(out, dense)
    dw = [torch.empty(K, N, dtype=dtype, device="cuda") for _ in range(2)]
    linear.gemm_linear_bwd(out, x, None, None, None, dw[0])
    linear.gemm_linear_bwd(dense, x.contiguous(), None, None, None, dw[1])
    assert same(*dw)
