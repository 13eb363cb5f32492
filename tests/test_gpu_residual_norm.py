"""The norms with the residual stream, forward and backward, against the formulas in 64 bits and against differences."""
import numpy as np
import pytest
import torch

from tests.block_ref import DTYPES, TINY, U, inside, per_token, residual_norm, rms, same

pytestmark = pytest.mark.gpu


def values(g, shape, dtype, sigma=1.0):
    return (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()


def close(got, want, bound, what=""):
    error = (got.double() - want).abs()
    assert torch.isfinite(error).all(), what
    worst = (error / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


def vectors(g, B, C, dtype, gate, post, wide):
    """gate: None, "channel", "sequence" or "sequence in wider rows"; wide: weights in 32 bits."""
    weight = torch.float32 if wide else dtype
    w = [(torch.rand(C, generator=g) + 0.5).to(weight).cuda() for _ in range(2)]
    found = None
    if gate == "channel":
        found = values(g, (C,), torch.float32 if wide else dtype)
    elif gate:
        found = inside((B, C), dtype, float("nan"), (0, 16 if gate.endswith("rows") else 0))[0].copy_(values(g, (B, C), dtype))
    return found, w[0] if post else None, w[1]


def layout(t, kind):
    """The same values as [B,N,C] on end, inside a larger tensor of NaN, or with sequences inside tokens."""
    B, N, C = t.shape
    if kind == "wide":
        return inside((B, N, C), t.dtype, float("nan"), (1, 2, 24))[0].copy_(t)
    if kind == "tokens first":
        return torch.empty(N, B, C, dtype=t.dtype, device="cuda").transpose(0, 1).copy_(t)
    return t


FORMS = [(None, False, 1.0, False, "on end"), ("channel", False, 0.75, True, "wide"), ("sequence", True, 1.0, False, "tokens first"),
         (None, True, -0.5, True, "on end"), ("channel", True, 1.0, False, "tokens first"), ("sequence in wider rows", False, 1.0, True, "wide")]
# channels on both sides of what a wave, two, four and eight hold with one, two, three and four vectors a lane; tokens in one and in many runs
SIZES = [(1, 1, 8), (2, 3, 64), (3, 37, 512), (2, 5, 520), (1, 129, 1032), (2, 70, 1544), (3, 9, 2056), (1, 7, 4096), (2, 2, 4104), (1, 3, 8200), (2, 1, 16384),
         (5, 1100, 72)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gate,post,alpha,wide,where", FORMS)
@pytest.mark.parametrize("B,N,C", SIZES)
def test_forward_and_backward_match_the_formulas(B, N, C, gate, post, alpha, wide, where, dtype):
    from paper_2403_16863_amd import norm
    g = torch.Generator().manual_seed(B + N + C)
    eps = 1e-5
    x, h, dy, dz = (layout(values(g, (B, N, C), dtype, s), where) for s in (2.0, 1.0, 1.0, 1.0))
    gate, post, pre = vectors(g, B, C, dtype, gate, post, wide)
    outs = [layout(torch.full((B, N, C), float("nan"), dtype=dtype, device="cuda"), where) for _ in range(4)]
    y, z, dx, dh = outs
    norm.residual_norm(x, h, y, z, gate, post, pre, alpha, eps)
    x64, h64, g64, p64, q64 = (None if t is None else t.double() for t in (x, h, gate, post, pre))
    want_y, want_z = residual_norm(x64, h64, g64, p64, q64, alpha, eps)
    # half a step of the result; in 32 bits a few roundings of the two terms of y, and a mean square that is C sums of one sign in a tree (2^-20)
    terms = alpha * x64.abs() + (want_y - alpha * x64).abs() if alpha > 0 else (alpha * x64).abs() + (want_y - alpha * x64).abs()
    close(y, want_y, U[dtype] * want_y.abs() + TINY[dtype] + 2.0 ** -20 * terms, "y")
    close(z, want_z, U[dtype] * want_z.abs() + TINY[dtype] + 2.0 ** -19 * q64 * rms(want_y, eps) * terms, "z")

    # backward, from the rounded y, as a program has it
    grads = [None if v is None else torch.full(v.shape, float("nan"), device="cuda") for v in (gate, post, pre)]
    norm.residual_norm_bwd(dy, dz, y, h, dx, dh, gate, post, pre, *grads, alpha, eps)
    y64, dy64, dz64 = y.double(), dy.double(), dz.double()
    r, gt = rms(y64, eps), per_token(g64)
    n, p = y64 * r, dz64 * q64
    D = dy64 + r * (p - n * (p * n).mean(-1, keepdim=True))
    size = dy64.abs() + r * (p.abs() + n.abs() * (p * n).abs().mean(-1, keepdim=True))      # what D is the sum of
    close(dx, alpha * D, U[dtype] * (alpha * D).abs() + TINY[dtype] + 2.0 ** -18 * abs(alpha) * size, "dx")
    G = D * gt
    n1 = h64 if post is None else h64 * rms(h64, eps)
    gsize = size * (gt.abs() if torch.is_tensor(gt) else gt)
    if post is None:
        want_h, hsize = G, gsize
    else:
        r1, p1, ps = rms(h64, eps), G * p64, gsize * p64
        want_h = r1 * (p1 - n1 * (p1 * n1).mean(-1, keepdim=True))
        hsize = r1 * (ps + n1.abs() * (ps * n1.abs()).mean(-1, keepdim=True))
    close(dh, want_h, U[dtype] * want_h.abs() + TINY[dtype] + 2.0 ** -17 * hsize, "dh")
    u = n1 if post is None else n1 * p64
    tokens = B * N
    for name, got, term, tsize in (("dgate", grads[0], D * u, size * u.abs()), ("dpost_weight", grads[1], G * n1, gsize * n1.abs()),
                                   ("dpre_weight", grads[2], dz64 * n, (dz64 * n).abs())):
        if got is None:
            continue
        over = 1 if got.dim() == 2 else (0, 1)
        # sums of as many terms in 32 bits, each off by 2^-17 of what it is made of
        close(got, term.sum(over), ((tokens + 8) * 2.0 ** -24 + 2.0 ** -17) * tsize.sum(over) + 1e-30, name)


@pytest.mark.parametrize("dtype", DTYPES)
def test_forms_with_parts_left_out(dtype):
    """Plain norm, stream alone, gradients of one output alone, and vectors' gradients left out."""
    from paper_2403_16863_amd import norm
    B, N, C = 2, 19, 264
    g = torch.Generator().manual_seed(7)
    x, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, "sequence", True, False)

    def new():
        return torch.full((B, N, C), float("nan"), dtype=dtype, device="cuda")
    y, z = new(), new()
    norm.residual_norm(x, h, y, z, gate, post, pre)
    alone = new()
    norm.residual_norm(x, h, alone, None, gate, post)
    assert same(alone, y)
    norm.residual_norm(x, h, None, alone, gate, post, pre)
    assert same(alone, z)
    plain = new()
    norm.residual_norm(x, None, None, plain, None, None, pre)
    _, want = residual_norm(x.double(), None, None, None, pre.double(), 1.0, 1e-6)
    close(plain, want, U[dtype] * want.abs() + TINY[dtype] + 2.0 ** -19 * want.abs())
    # without dz: what comes back along the stream alone;  without dy: what comes back through the norm alone
    dx, dh, whole = new(), new(), [torch.empty(s, device="cuda") for s in ((B, C), (C,), (C,))]
    norm.residual_norm_bwd(dy, None, None, h, dx, dh, gate, post, None, whole[0], whole[1])
    assert same(dx, dy)
    r1 = rms(h.double(), 1e-6)
    n1 = h.double() * r1
    p1 = dy.double() * gate.double()[:, None] * post.double()
    want = r1 * (p1 - n1 * (p1 * n1).mean(-1, keepdim=True))
    close(dh, want, U[dtype] * want.abs() + TINY[dtype] + 2.0 ** -17 * r1 * (p1.abs() + n1.abs() * (p1 * n1).abs().mean(-1, keepdim=True)))
    zero = torch.zeros_like(dy)
    a, b = [new(), new()], [new(), new()]
    norm.residual_norm_bwd(None, dz, y, h, *a, gate, post, pre)
    norm.residual_norm_bwd(zero, dz, y, h, *b, gate, post, pre, *whole)
    assert same(a[0], b[0]) and same(a[1], b[1])
    for i in range(3):                                                  # each vector's gradient alone, and none
        some = [None] * 3
        some[i] = torch.empty_like(whole[i])
        norm.residual_norm_bwd(None, dz, y, h, *b, gate, post, pre, *some)
        assert same(some[i], whole[i]) and same(a[1], b[1])
    only = new()
    norm.residual_norm_bwd(None, dz, y, h, None, only, gate, post, pre)
    assert same(only, a[1])
    norm.residual_norm_bwd(None, dz, y, None, only, None, None, None, pre, None, None, whole[2])       # the plain norm's
    assert same(only, a[0])
    # neither gate nor norm behind the block: dh is D itself, and h is not looked at
    norm.residual_norm_bwd(dy, dz, y, None, dx, dh, None, None, pre, alpha=1.0)
    assert same(dx, dh)


def test_gradients_match_differences():
    from paper_2403_16863_amd import norm
    B, N, C, eps, alpha, dtype = 2, 3, 64, 0.25, 0.75, torch.float16
    g = torch.Generator().manual_seed(8)
    x, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, "sequence", True, True)
    y, z, dx, dh = (torch.empty_like(x) for _ in range(4))
    grads = [torch.empty(v.shape, device="cuda") for v in (gate, post, pre)]
    norm.residual_norm(x, h, y, z, gate, post, pre, alpha, eps)
    norm.residual_norm_bwd(dy, dz, y, h, dx, dh, gate, post, pre, *grads, alpha, eps)
    rng = np.random.default_rng(1)
    at = [t.double() for t in (x, h, gate, post, pre)]
    for _ in range(8):
        v = [torch.from_numpy(rng.standard_normal(t.shape)).cuda() for t in at]
        e = 1e-6

        def loss(a):
            yy, zz = residual_norm(*(t + a * d for t, d in zip(at, v)), alpha, eps)
            return ((yy * dy.double()).sum() + (zz * dz.double()).sum()).item()
        slope = (loss(e) - loss(-e)) / (2 * e)
        parts = [t.double() * d for t, d in zip((dx, dh, *grads), v)]
        # dx and dh are rounded to binary16, and the gradients are taken at the rounded y, half a step off in every channel (its change of D: twice
        # the norm's slope of about 2): four deviations
        tol = 4 * 2.0 ** -11 * (sum((q ** 2).sum().item() for q in parts) * 8) ** 0.5 + 1e-4
        assert abs(sum(q.sum().item() for q in parts) - slope) <= tol


@pytest.mark.parametrize("C", [264, 4096])
def test_outputs_in_the_inputs_memory(C):
    from paper_2403_16863_amd import norm
    B, N, dtype = 2, 33, torch.bfloat16
    g = torch.Generator().manual_seed(9)
    x, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, "channel", True, True)
    y, z, dx, dh = (torch.empty_like(x) for _ in range(4))
    norm.residual_norm(x, h, y, z, gate, post, pre)
    stream, block = x.clone(), h.clone()
    norm.residual_norm(stream, block, stream, block, gate, post, pre)              # the stream in place, z where h was
    assert same(stream, y) and same(block, z)
    norm.residual_norm_bwd(dy, dz, y, h, dx, dh, gate, post, pre)
    for a, b in ((0, 1), (1, 0), (2, 3), (3, 2)):                                  # of dy, dz, y, h
        mine = [t.clone() for t in (dy, dz, y, h)]
        norm.residual_norm_bwd(*mine, mine[a], mine[b], gate, post, pre)
        assert same(mine[a], dx) and same(mine[b], dh)
    joint = torch.cat((x, h, torch.zeros_like(x)), -1)                             # side by side in wider rows
    norm.residual_norm(joint[..., :C], joint[..., C:2 * C], joint[..., 2 * C:], None, gate, post)
    assert same(joint[..., 2 * C:], y) and same(joint[..., :C], x)


def test_tokens_of_zeros_infinities_and_nan_stay_alone():
    from paper_2403_16863_amd import norm
    B, N, C, dtype = 1, 40, 520, torch.float16
    g = torch.Generator().manual_seed(10)
    x, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, None, True, True)
    want = [torch.empty_like(x) for _ in range(4)]
    norm.residual_norm(x, h, *want[:2], gate, post, pre)
    norm.residual_norm_bwd(dy, dz, want[0], h, *want[2:], gate, post, pre)
    x[0, 3], h[0, 3] = 0, 0                                                        # a padded token: zeros, not NaN
    x[0, 9, 5], h[0, 21, 519] = float("nan"), float("inf")
    x[0, 30] = 65504.0                                                             # squares beyond binary16, not beyond 32 bits
    got = [torch.empty_like(x) for _ in range(4)]
    norm.residual_norm(x, h, *got[:2], gate, post, pre)
    norm.residual_norm_bwd(dy, dz, got[0], h, *got[2:], gate, post, pre)
    keep = torch.ones(N, dtype=torch.bool, device="cuda")
    keep[[3, 9, 21, 30]] = False
    for a, b in zip(got, want):
        assert same(a[:, keep], b[:, keep])
    assert (got[0][0, 3] == 0).all() and (got[1][0, 3] == 0).all()
    assert torch.isnan(got[1][0, 9]).all() and torch.isnan(got[0][0, 9, 5]) and torch.isfinite(got[0][0, 9, :5]).all()
    assert torch.isnan(got[0][0, 21, 519]) and torch.isfinite(got[1][0, 30]).all()
    close(got[1][0, 30], torch.full((C,), 1.0, device="cuda").double() * pre.double(), 2.0 ** -9 * pre.double())


@pytest.mark.parametrize("gate", ["channel", "sequence"])
def test_the_same_every_time_on_streams_and_from_graphs(gate):
    from paper_2403_16863_amd import norm
    B, N, C, dtype = 3, 700, 520, torch.bfloat16
    g = torch.Generator().manual_seed(11)
    y, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, gate, True, False)

    def fresh():
        return [torch.full((B, N, C), float("nan"), dtype=dtype, device="cuda") for _ in range(2)] + \
            [torch.full(v.shape, float("nan"), device="cuda") for v in (gate, post, pre)]

    def call(o, **more):
        norm.residual_norm_bwd(dy, dz, y, h, o[0], o[1], gate, post, pre, *o[2:], **more)
        return o
    want = call(fresh())
    assert all(same(a, b) for a, b in zip(call(fresh()), want))
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="workspace"):
        call(fresh(), stream=side.cuda_stream)
    space, outs = torch.empty(norm.residual_norm_bwd_workspace(B, N, C, gate.dim() == 2), dtype=torch.uint8, device="cuda"), fresh()
    torch.cuda.synchronize()
    call(outs, stream=side.cuda_stream, workspace=space)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(outs, want))
    graphs, outs = [], [fresh(), fresh()]
    for o in outs:
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


def test_many_sequences_with_a_gate_each():
    """More sequences than workgroups: each goes through several, and adds what post_weight's gradient takes from them."""
    from paper_2403_16863_amd import norm
    B, N, C, dtype = 1300, 2, 64, torch.float16
    g = torch.Generator().manual_seed(12)
    y, h, dy, dz = (values(g, (B, N, C), dtype) for _ in range(4))
    gate, post, pre = vectors(g, B, C, dtype, "sequence", True, True)
    dx, dh = torch.empty_like(y), torch.empty_like(y)
    grads = [torch.full(v.shape, float("nan"), device="cuda") for v in (gate, post, pre)]
    norm.residual_norm_bwd(dy, dz, y, h, dx, dh, gate, post, pre, *grads)
    y64, h64 = y.double(), h.double()
    r = rms(y64, 1e-6)
    n, p = y64 * r, dz.double() * pre.double()
    D = dy.double() + r * (p - n * (p * n).mean(-1, keepdim=True))
    size = dy.double().abs() + r * (p.abs() + n.abs() * (p * n).abs().mean(-1, keepdim=True))
    n1 = h64 * rms(h64, 1e-6)
    for got, term, tsize, over in ((grads[0], D * n1 * post.double(), size * (n1 * post.double()).abs(), 1),
                                   (grads[1], D * gate.double()[:, None] * n1, size * (gate.double()[:, None] * n1).abs(), (0, 1)),
                                   (grads[2], dz.double() * n, (dz.double() * n).abs(), (0, 1))):
        close(got, term.sum(over), ((B * N + 8) * 2.0 ** -24 + 2.0 ** -17) * tsize.sum(over))


def test_tokens_far_behind_32_bits():
    from paper_2403_16863_amd import norm
    B, N, C, dtype = 2, 3, 64, torch.float16
    far = (1 << 31) + 1024                                                         # elements
    if torch.cuda.mem_get_info()[0] < 5 * far * 2 + (1 << 30):
        pytest.skip("needs 22 GB")
    g = torch.Generator().manual_seed(13)
    x, h = values(g, (B, N, C), dtype), values(g, (B, N, C), dtype)
    pre = torch.ones(C, device="cuda")
    want = [torch.empty_like(x) for _ in range(2)]
    norm.residual_norm(x, h, *want, None, None, pre)
    whole = torch.empty(2, far + N * C, dtype=dtype, device="cuda")
    a, b = (torch.as_strided(t, (B, N, C), (far, C, 1)) for t in whole)
    norm.residual_norm(a.copy_(x), b.copy_(h), a, b, None, None, pre)
    assert same(a, want[0]) and same(b, want[1])
