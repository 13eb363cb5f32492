"""The 4-bit cache and the attention over it against the definitions in 64 bits (tests/kv4_ref.py)."""
import numpy as np
import pytest
import torch

from tests import kv4_ref as R

pytestmark = pytest.mark.gpu

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.float16, torch.bfloat16]


def f64(t):
    return t.double().cpu().numpy()


def tables_for(d, rows, seed=0):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, d, 2) / d)
    return torch.from_numpy(np.cos(a)).float().cuda(), torch.from_numpy(np.sin(a)).float().cuda()


def rotated32(k, c, s, interleaved):
    """The rotation as the elementary operations in 32 bits, which the codes are defined by."""
    a, b = (k[..., 0::2], k[..., 1::2]) if interleaved else k.chunk(2, -1)
    u, w = a * c - b * s, b * c + a * s
    return torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)


def special_values(x):
    """Ties, signed zeros, saturating, tiny, infinite and NaN values into a tensor [T, heads, d]."""
    with torch.no_grad():
        x[0, 0, :32] = torch.tensor([7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -7] * 2)
        x[0, 0, 32:64] = torch.tensor([0.0, -0.0] * 16)
        if x.shape[0] > 3:
            x[1, -1, :32] = 2.0 ** -24
            x[1, -1, 32:64] = torch.tensor([60000.0, -1.0] * 16)
            x[2, 0, 3] = float("inf")
            x[2, 0, 40] = float("nan")
            x[3, 0, 5] = -float("inf")
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,heads,page,how", [(1, 1, 16, "none"), (5, 3, 16, "half"), (33, 2, 64, "pairs"), (70, 1, 32, "half")])
def test_append_writes_the_defined_bytes_and_no_others(T, heads, page, how, d, dtype):
    g = torch.Generator().manual_seed(T * d)
    kv = torch.randn(T, 2 * heads + 1, d + 8, generator=g)
    kv[..., :d] = special_values(kv[..., :d])
    kv = kv.to(dtype).cuda()
    k, v = kv[:, :heads, :d], kv[:, heads:2 * heads, :d]          # strides of a wider projection
    pages = T // page + 3
    cache = torch.randint(0, 256, (pages, heads, page, d + d // 16), generator=g, dtype=torch.uint8).cuda()
    want = cache.cpu().numpy().copy()
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    slots[T // 2] = -1 if T > 1 else slots[0]
    if T > 4:
        slots[4] = pages * page
    c, s = tables_for(d, 40)
    positions = torch.randint(0, 40, (T,), generator=g).int().cuda()
    rotated = k.float()
    if how == "none":
        from paper_2403_16863_amd import kv4
        kv4.kv4_append(k, v, cache, slots.cuda())
    else:
        from paper_2403_16863_amd import kv4
        if T > 6:
            positions[6] = 40                                      # behind the table: the key is NaN
        kv4.kv4_append(k, v, cache, slots.cuda(), c, s, positions, interleaved=how == "pairs")
        at = positions.long().clamp(max=39)
        rotated = rotated32(rotated, c[at][:, None], s[at][:, None], how == "pairs")
        if T > 6:
            rotated[6] = float("nan")
    rotated, v64 = f64(rotated), f64(v)
    for t in range(T):
        if 0 <= int(slots[t]) < pages * page:
            for h in range(heads):
                R.put(want, int(slots[t]), h, rotated[t, h], v64[t, h])
    assert np.array_equal(cache.cpu().numpy(), want)
    # and back
    kr, vr = torch.empty(T, heads, d, dtype=dtype, device="cuda"), torch.empty(T, heads, d, dtype=dtype, device="cuda")
    kv4.kv4_read(cache, slots.cuda(), kr, vr)
    kw, vw = R.values(want)
    for t in range(T):
        n = int(slots[t])
        inside = 0 <= n < pages * page
        for got, all_ in ((kr, kw), (vr, vw)):
            expect = all_[n // page, :, n % page] if inside else np.zeros((heads, d))
            assert np.array_equal(f64(got[t]), expect, equal_nan=True), t
    only = torch.empty_like(vr)
    kv4.kv4_read(cache, slots.cuda(), v=only)
    assert torch.equal(only.view(torch.int16), vr.view(torch.int16))


def fill(pages, heads, page, d, seed, scale=1.0):
    """A cache of random values, made by the append itself (held to the definition above), from 0xff bytes."""
    from paper_2403_16863_amd import kv4
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = torch.full(kv4.kv4_cache_shape(pages, heads, page, d), 255, dtype=torch.uint8, device="cuda")
    k, v = (torch.randn(pages * page, heads, d, device="cuda", generator=g).mul_(scale).half() for _ in range(2))
    kv4.kv4_append(k, v, cache, torch.arange(pages * page, dtype=torch.int32, device="cuda"))
    return cache


def check(out, lse, want, dtype, scores=1.0, rows=None):
    """Rounding the result costs u, rounding the probabilities to binary16 2^-11 of sum p |v|; fp32 terms: an exponential's argument is
    off by at most 2^-21 times the largest score (in powers of two), which scales p, and d + keys additions."""
    o, l, spread = want
    rows = slice(None) if rows is None else rows
    o, l, spread, out, lse = o[rows], l[rows], spread[rows], f64(out)[rows], f64(lse)[rows]
    small = 2.0 ** -20 * max(1.0, scores) * 4
    tol = U[dtype] * np.abs(o) + (2.0 ** -11 + small) * spread + 2.0 ** -24
    assert (np.abs(out - o) <= tol).all(), float((np.abs(out - o) / tol).max())
    assert np.array_equal(np.isinf(lse), np.isinf(l)) and np.array_equal(lse[np.isinf(l)], l[np.isinf(l)])
    f = np.isfinite(l)
    assert (np.abs(lse[f] - l[f]) <= small * np.maximum(1, np.abs(l[f]))).all()


CASES = [
    # lens, queries, H, heads, d, page, causal
    ([1], [1], 1, 1, 64, 16, True),
    ([0, 1, 16, 17], [1, 1, 1, 1], 8, 2, 128, 16, True),
    ([31, 32, 33, 15], [1, 2, 1, 3], 4, 4, 64, 16, True),
    ([127, 128, 129, 400], [1, 1, 1, 1], 5, 1, 128, 32, True),
    ([300, 5, 0, 129], [4, 9, 3, 0], 6, 2, 64, 64, True),          # more queries than keys, none at all
    ([200, 333], [7, 11], 6, 2, 128, 16, True),                    # rows beyond 16 and 32
    ([65, 260], [40, 70], 3, 1, 64, 128, True),                    # several row blocks
    ([65, 260, 40], [40, 70, 1], 2, 1, 128, 16, False),            # every key visible
    ([700, 3, 1100], [1, 1, 1], 16, 1, 128, 16, True),             # one head for all
    ([350], [350], 4, 2, 64, 64, True),                            # a fresh prompt
    ([513], [300], 8, 2, 128, 32, True),                           # a chunk
    ([640], [260], 4, 4, 128, 64, False),
]


def setup(case, dtype, seed=0, sigma=1.5):
    lens, nqs, H, heads, d, page, causal = case
    g = torch.Generator().manual_seed(seed)
    width = max(1, -(-max(lens) // page)) + 1
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 2
    perm = torch.randperm(pages, generator=g).int()
    tables = torch.full((len(lens), width), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        tables[b, :n] = perm[at:at + n]
        at += n
    cache = fill(pages, heads, page, d, seed)
    cu = [0]
    for n in nqs:
        cu.append(cu[-1] + n)
    q = (torch.randn(cu[-1], H, d, generator=g) * sigma).to(dtype).cuda()
    return dict(q=q, cache=cache, tables=tables.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda(),
                cu=torch.tensor(cu, dtype=torch.int32).cuda(), max_q=max(nqs), causal=causal, scale=d ** -0.5)


def run(s, workspace=None, stream=None, out=None, lse=None):
    from paper_2403_16863_amd import kv4
    out = torch.full_like(s["q"], float("nan")) if out is None else out
    lse = torch.full(s["q"].shape[:2], float("nan"), device="cuda") if lse is None else lse
    kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], out, lse, s["causal"], s["scale"], s["cu"], s["max_q"], workspace, stream)
    return out, lse


def reference(s):
    return R.attention(f64(s["q"]), R.values(s["cache"].cpu().numpy()), s["tables"].cpu().numpy(), s["lens"].cpu().numpy(),
                       s["cu"].cpu().numpy(), s["causal"], s["scale"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[0])) + f"-q{max(c[1])}-{c[2]}on{c[3]}-d{c[4]}")
def test_attention_matches_the_definition_with_and_without_runs(case, dtype):
    s = setup(case, dtype)
    want = reference(s)
    whole = run(s)
    check(*whole, want, dtype, scores=60)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    uncut = run(s, stream=side.cuda_stream)                        # no workspace there: keys in one run
    torch.cuda.synchronize()
    check(*uncut, want, dtype, scores=60)
    again = run(s)
    assert torch.equal(again[0].view(torch.int16), whole[0].view(torch.int16)) and torch.equal(again[1], whole[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_without_cu_q_every_sequence_has_as_many_queries(dtype):
    from paper_2403_16863_amd import kv4
    s = setup(([40, 90, 17], [2, 2, 2], 4, 2, 64, 16, True), dtype)
    want = run(s)
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], out, lse, True, s["scale"])
    assert torch.equal(out.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])


def test_many_sequences_and_rows_of_nobody():
    lens = [1 + (37 * i) % 90 for i in range(150)]
    s = setup((lens, [1] * 150, 4, 2, 64, 16, True), torch.float16)
    want = reference(s)
    check(*run(s), want, torch.float16, scores=60)
    pad = torch.zeros(5, 4, 64, dtype=torch.float16, device="cuda")
    s["q"], s["cu"] = torch.cat((pad, s["q"], pad)), s["cu"] + 5
    out, lse = run(s)
    check(out[5:155], lse[5:155], want, torch.float16, scores=60)
    for x in (out, lse):
        assert torch.isnan(x[:5]).all() and torch.isnan(x[155:]).all()


def random_case(B, most, most_q, H, heads, d, seed, empty=4):
    """Lengths of all sizes, some of them and some numbers of queries zero."""
    r = np.random.default_rng(seed)
    lens = [0 if r.integers(empty + 6) == 0 else int(most ** r.uniform(0, 1)) for _ in range(B)]
    nqs = [0 if r.integers(empty) == 0 else int(r.integers(1, most_q + 1)) for _ in range(B)]
    lens[B // 2], nqs[B // 2] = most, most_q
    return lens, nqs, H, heads, d, 16, True


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,most,most_q,H,heads,d", [
    (70, 2600, 1, 4, 2, 64), (130, 2600, 2, 4, 1, 128),            # ranges over more sequences than a wave has lanes
    (9, 4100, 3, 6, 2, 128), (9, 4100, 9, 6, 2, 64),               # ranges that end inside, at and behind sequences, some without rows
    (5, 3000, 50, 4, 2, 64), (6, 2300, 90, 4, 1, 128),             # the same of many rows
    (66, 300, 40, 2, 1, 64), (64, 200, 60, 3, 1, 128), (3, 500, 150, 2, 2, 64),     # whole row blocks, in layers and not
])
def test_unequal_sequences(B, most, most_q, H, heads, d, dtype):
    s = setup(random_case(B, most, most_q, H, heads, d, B + d), dtype, seed=B)
    want = reference(s)
    check(*run(s), want, dtype, scores=60)
    s["causal"] = False
    check(*run(s), reference(s), dtype, scores=60)


def test_lengths_at_the_edges_of_a_range():
    """The shortest ranges, with lengths around their ends: every piece of a row has to be joined, once."""
    for d, q in ((64, 1), (128, 40)):
        for n in (2049, 2080, 2081, 2112, 2500, 3000, 3500, 4096):
            s = setup(([n], [q], 1, 1, d, 64, True), torch.float16, seed=n)
            check(*run(s), reference(s), torch.float16, scores=60)


def test_pages_outside_the_cache_are_not_seen_and_lengths_are_limited():
    s = setup(([100, 100, 100], [3, 3, 3], 4, 2, 64, 16, True), torch.float16)
    s["tables"][0, 1] = -1
    s["tables"][1, 0] = s["cache"].shape[0]
    s["tables"][2] = torch.iinfo(torch.int32).max                  # no key at all
    check(*run(s), reference(s), torch.float16, scores=60)
    s["tables"][:] = torch.arange(3 * 8, device="cuda").view(3, 8) % s["cache"].shape[0]
    s["lens"][:] = torch.tensor([2 ** 31 - 1, -5, 128])
    check(*run(s), reference(s), torch.float16, scores=60)


def test_one_page_may_belong_to_several_sequences():
    s = setup(([48, 48], [2, 2], 2, 1, 128, 16, True), torch.bfloat16)
    s["tables"][1] = s["tables"][0]
    check(*run(s), reference(s), torch.bfloat16, scores=60)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq", [4, 100])
def test_nan_among_values_and_keys_stays_with_the_rows_that_see_it(d, nq):
    s = setup(([130], [nq], 2, 1, d, 16, True), torch.float16)
    cache, tables = s["cache"].cpu().numpy(), s["tables"].cpu().numpy()
    for what, key in ((4, 128), (3, 129)):                         # the scale of a value block, then of a key block
        bad = cache.copy()
        place = R.token_place(d, key % 16, 33)
        bad[tables[0, key // 16], 0].reshape(-1)[place[what]] = 255
        s["cache"] = torch.from_numpy(bad).cuda()
        out, lse = run(s)
        s["cache"] = torch.from_numpy(cache).cuda()
        want = reference(s)
        seen = np.array([key <= 130 - nq + i for i in range(nq)])
        check(out, lse, want, torch.float16, scores=60, rows=~seen)
        got = f64(out)[seen]
        assert np.isnan(got[..., 32:64]).all()
        if what == 3:
            assert np.isnan(got).all() and np.isnan(f64(lse)[seen]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_queries_of_any_magnitude(dtype):
    s = setup(([64], [6], 1, 1, 64, 16, False), dtype)
    s["scale"] = 1.0
    with torch.no_grad():
        s["q"][0] = 0
        s["q"][1] *= 2.0 ** -10
        s["q"][2, 0, :] = 2.0 ** -14
        if dtype == torch.bfloat16:
            s["q"][3] *= 1e-30
    out, lse = run(s)
    check(out, lse, reference(s), dtype, scores=300)
    with torch.no_grad():
        s["q"][4, 0, 7], s["q"][5, 0, 9] = float("inf"), float("nan")
    out, lse = run(s)
    assert torch.isnan(out[4:]).all() and torch.isnan(lse[4:]).all() and not torch.isnan(out[:4]).any()


def test_a_raised_maximum_late_in_a_long_row():
    """Keys that grow along the sequence: every tile raises the reference."""
    from paper_2403_16863_amd import kv4
    n, d = 2000, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = torch.zeros(kv4.kv4_cache_shape(125, 1, 16, d), dtype=torch.uint8, device="cuda")
    q = torch.ones(1, 4, d, device="cuda", dtype=torch.bfloat16)
    k = (torch.arange(n, device="cuda")[:, None, None] * 0.02 + torch.randn(n, 1, d, device="cuda", generator=g) * 0.1).bfloat16()
    v = torch.randn(n, 1, d, device="cuda", generator=g).bfloat16()
    kv4.kv4_append(k, v, cache, torch.arange(n, device="cuda", dtype=torch.int32))
    s = dict(q=q, cache=cache, tables=torch.arange(125, device="cuda", dtype=torch.int32)[None], lens=torch.tensor([n], dtype=torch.int32).cuda(),
             cu=torch.tensor([0, 1], dtype=torch.int32).cuda(), max_q=1, causal=True, scale=d ** -0.5)
    check(*run(s), reference(s), torch.bfloat16, scores=700)


def test_offsets_beyond_32_bits():
    from paper_2403_16863_amd import kv4
    heads, page, d = 8, 64, 128
    pages = (5 << 30) // (heads * page * (d + d // 16))
    cache = torch.empty(kv4.kv4_cache_shape(pages, heads, page, d), dtype=torch.uint8, device="cuda")
    n, g = 100, torch.Generator(device="cuda").manual_seed(5)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    slots = (table[0, j // page] * page + j % page).int()
    k, v = (torch.randn(n, heads, d, device="cuda", generator=g).half() for _ in range(2))
    kv4.kv4_append(k, v, cache, slots)
    q = torch.randn(1, 16, d, device="cuda", generator=g).half()
    s = dict(q=q, cache=cache, tables=table, lens=torch.tensor([n], dtype=torch.int32).cuda(), cu=torch.tensor([0, 1], dtype=torch.int32).cuda(),
             max_q=1, causal=True, scale=d ** -0.5)
    got = run(s)
    s["cache"], s["tables"] = cache[[pages - 1, pages - 2]].contiguous(), torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    check(*got, reference(s), torch.float16, scores=60)


def test_a_captured_step_meets_new_lengths_at_each_replay():
    """Append and attention in one graph: lengths, slots and tokens change between replays, with eager work beside it, and a
    second graph of the same buffers."""
    from paper_2403_16863_amd import kv4
    B, H, heads, d, page, width = 3, 8, 2, 64, 16, 40
    cache = fill(B * width, heads, page, d, 7)
    tables = torch.randperm(B * width, generator=torch.Generator().manual_seed(1)).int().view(B, width).cuda()
    lens, slots = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    positions = torch.zeros(B, dtype=torch.int32, device="cuda")
    c, s = tables_for(d, width * page)
    q, k, v = (torch.randn(B, n, d, device="cuda").half() for n in (H, heads, heads))
    outs = [(torch.empty_like(q), torch.empty(B, H, device="cuda")) for _ in range(3)]

    def step(out, lse):
        kv4.kv4_append(k, v, cache, slots, c, s, positions)
        kv4.kv4_attn(q, cache, tables, lens, out, lse, True, d ** -0.5)
    step(*outs[0])
    torch.cuda.synchronize()
    graphs = []
    for i in (1, 2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            step(*outs[i])
        graphs.append(graph)
    g = torch.Generator(device="cuda").manual_seed(11)
    for at in ([0, 5, 600], [1, 6, 601], [300, 127, 17], [639, 0, 255]):
        n = torch.tensor(at, device="cuda")
        lens.copy_(n + 1)
        positions.copy_(n)
        slots.copy_(tables.gather(1, (n // page)[:, None]).squeeze(1) * page + n % page)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda", generator=g))
        step(*outs[0])
        torch.cuda.synchronize()
        for graph, (out, lse) in zip(graphs, outs[1:]):
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), outs[0][0].view(torch.int16)) and torch.equal(lse, outs[0][1])


def test_two_streams_at_once():
    cases = [setup(([3000, 2500], [1, 1], 8, 2, 128, 16, True), torch.float16, seed=i) for i in range(2)]
    alone = [run(s) for s in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for s, stream in zip(cases, streams):
        with torch.cuda.stream(stream):
            for _ in range(20):
                last = run(s)
            got.append(last)
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1])


def test_given_workspace_and_small_ones():
    from paper_2403_16863_amd import kv4
    s = setup(([3000], [1], 8, 2, 128, 16, True), torch.float16)
    B, width = s["tables"].shape
    need = kv4.kv4_attn_workspace(1, B, 8, 2, 128, 16, width, 1)
    assert need > 0
    want = run(s)
    got = run(s, workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(got[0].view(torch.int16), want[0].view(torch.int16)) and torch.equal(got[1], want[1])
    with pytest.raises(ValueError, match="workspace"):
        run(s, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_layer_from_projection_to_attention(dtype):
    """Norms and rotation, the cache, and attention over it, for a prompt and the tokens after it, as a layer uses them."""
    from paper_2403_16863_amd import kv4, rope
    H, heads, d, page, n, later = 6, 2, 128, 16, 45, 3
    g = torch.Generator(device="cuda").manual_seed(2)
    qw, kw = (torch.rand(d, device="cuda", generator=g).add_(0.5).to(dtype) for _ in range(2))
    c, s = tables_for(d, n + later)
    cache = torch.full(kv4.kv4_cache_shape(5, heads, page, d), 255, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[3, 0, 4, 1]], dtype=torch.int32, device="cuda")
    outs, qs = [], []
    for first, m in ((0, n), *((n + i, 1) for i in range(later))):
        qkv = torch.randn(1, m, H + 2 * heads, d, device="cuda", generator=g).to(dtype)
        positions = torch.arange(first, first + m, device="cuda", dtype=torch.int32)
        q, k = torch.empty(1, m, H, d, device="cuda", dtype=dtype), torch.empty(1, m, heads, d, device="cuda", dtype=dtype)
        rope.qk_norm_rope(qkv[:, :, :H], qkv[:, :, H:H + heads], q, k, c, s, positions[None], qw, kw)
        slots = (table[0, positions.long() // page] * page + positions % page).int()
        kv4.kv4_append(k[0], qkv[0, :, H + heads:], cache, slots)
        out, lse = torch.empty(m, H, d, device="cuda", dtype=dtype), torch.empty(m, H, device="cuda")
        kv4.kv4_attn(q[0], cache, table, torch.tensor([first + m], device="cuda", dtype=torch.int32), out, lse, True, d ** -0.5)
        outs.append((out, lse))
        qs.append(q[0])
    # one causal pass over all tokens and the cache as it is now
    want = R.attention(f64(torch.cat(qs)), R.values(cache.cpu().numpy()), table.cpu().numpy(), [n + later], [0, n + later], True, d ** -0.5)
    check(torch.cat([o for o, _ in outs]), torch.cat([l for _, l in outs]), want, dtype, scores=60)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [([3000, 40, 0, 2500], [300, 30, 5, 256], 8, 2, 64, 16, True), ([2300, 2100], [257, 3], 8, 1, 128, 32, True),
                                  ([2500], [270], 4, 1, 128, 64, False)], ids=["four", "two", "all keys"])
def test_many_rows_over_long_caches(case, dtype):
    """More than a thousand rows to a sequence and head: blocks of 256 rows, cut and not, and pages that are not there."""
    s = setup(case, dtype)
    s["tables"][0, 3] = -1
    want = reference(s)
    check(*run(s), want, dtype, scores=60)
    uncut = run(s, stream=torch.cuda.Stream().cuda_stream)
    torch.cuda.synchronize()
    check(*uncut, want, dtype, scores=60)


@pytest.mark.parametrize("d", [64, 128])
def test_nan_in_a_long_cache_of_many_rows(d):
    n, nq, key = 2200, 600, 2130
    s = setup(([n], [nq], 2, 1, d, 16, True), torch.float16)
    cache = s["cache"].cpu().numpy()
    want = reference(s)
    for what in (4, 3):                                            # the scale of a value block, then of a key block
        bad = cache.copy()
        bad[int(s["tables"][0, key // 16]), 0].reshape(-1)[R.token_place(d, key % 16, 33)[what]] = 255
        s["cache"] = torch.from_numpy(bad).cuda()
        out, lse = run(s)
        seen = np.array([key <= n - nq + i for i in range(nq)])
        check(out, lse, want, torch.float16, scores=60, rows=~seen)
        got = f64(out)[seen]
        assert np.isnan(got[..., 32:64]).all() and (what == 4 or (np.isnan(got).all() and np.isnan(f64(lse)[seen]).all()))


@pytest.mark.parametrize("d", [64, 128])
def test_two_groups_of_waves_to_a_row_block(d):
    """A few prompts of odd and even numbers of tiles, pages that are not there, and a NaN in either group's tiles."""
    s = setup(([700, 64, 129, 1, 900], [100, 64, 50, 7, 60], 4, 2, d, 16, True), torch.bfloat16)
    s["tables"][4, 5] = -1
    check(*run(s), reference(s), torch.bfloat16, scores=60)
    n, nq = 700, 100
    s = setup(([n], [nq], 2, 1, d, 16, True), torch.float16)
    cache = s["cache"].cpu().numpy()
    want = reference(s)
    for what, key in ((4, 630), (4, 650), (3, 630), (3, 650)):     # of a value block, then of a key block, in tiles 9 and 10
        bad = cache.copy()
        bad[int(s["tables"][0, key // 16]), 0].reshape(-1)[R.token_place(d, key % 16, 33)[what]] = 255
        s["cache"] = torch.from_numpy(bad).cuda()
        out, lse = run(s)
        seen = np.array([key <= n - nq + i for i in range(nq)])
        check(out, lse, want, torch.float16, scores=60, rows=~seen)
        got = f64(out)[seen]
        assert np.isnan(got[..., 32:64]).all() and (what == 4 or (np.isnan(got).all() and np.isnan(f64(lse)[seen]).all()))
