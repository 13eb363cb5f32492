"""The attention over the 4-bit cache where its numbers are far apart, against the definition in 64 bits (tests/kv4_ref.py): each form of the
kernel, cut into ranges and not."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_ref as R
from tests.test_gpu_kv4 import DTYPES, U, f64

pytestmark = pytest.mark.gpu

# (keys, queries, page): one query head of d = 64 to a head of the cache, so queries are a segment's rows
FORMS = {
    "16 waves": (1500, 1, 16), "one row": (5000, 1, 16), "sixteen rows": (2600, 16, 16), "thirty rows": (2600, 30, 16),
    "thirty rows, short": (700, 30, 64), "two groups": (900, 100, 16), "many rows, short": (300, 100, 16), "many rows": (2600, 100, 32),
    "256 rows": (2500, 1100, 64),
}


def cache_of(k, v, page):
    """A cache of the given keys and values [n, d] in one head, in the order of its pages."""
    from paper_2403_16863_amd import kv4
    n, d = k.shape
    pages = -(-n // page)
    cache = torch.zeros(kv4.kv4_cache_shape(pages, 1, page, d), dtype=torch.uint8, device="cuda")
    kv4.kv4_append(k[:, None].half().cuda(), v[:, None].half().cuda(), cache, torch.arange(n, dtype=torch.int32, device="cuda"))
    return cache, torch.arange(pages, dtype=torch.int32, device="cuda")[None]


def attend(q, cache, tables, n, scale, cut):
    """out, lse of queries q [T, 1, d] of one sequence; without scratch memory where `cut` is false."""
    from paper_2403_16863_amd import kv4
    T = q.shape[0]
    out, lse = torch.full_like(q, float("nan")), torch.full((T, 1), float("nan"), device="cuda")
    lens, cu = torch.tensor([n], dtype=torch.int32).cuda(), torch.tensor([0, T], dtype=torch.int32).cuda()
    if cut:
        kv4.kv4_attn(q, cache, tables, lens, out, lse, True, scale, cu, T)
    else:                                                          # a stream that torch does not know: no memory taken
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        kv4.kv4_attn(q, cache, tables, lens, out, lse, True, scale, cu, T, stream=side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    return f64(out), f64(lse)


def defined(q, cache, tables, n, scale):
    return R.attention(f64(q), R.values(cache.cpu().numpy()), tables.cpu().numpy(), [n], [0, q.shape[0]], True, scale)


@pytest.mark.parametrize("cut", [True, False], ids=["cut", "uncut"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", FORMS)
def test_keys_far_below_the_largest_count(form, dtype, cut):
    """Every 32nd key has the largest score and the value 0; the others are 9 to 25 powers of two below it, and all of the output."""
    n, rows, page = FORMS[form]
    g = torch.Generator().manual_seed(n)
    for nats in (6.5, 9.8, 13.9, 17.5):
        k, v = torch.zeros(n, 64), torch.randint(1, 7, (n, 64), generator=g) * 4096.0
        k[::32, 0], v[::32] = 4, 0
        cache, tables = cache_of(k, v, page)
        q = torch.zeros(rows, 1, 64)
        q[:, 0, 0] = 1
        q = q.to(dtype).cuda()
        scale = nats / 4
        out, lse = attend(q, cache, tables, n, scale, cut)
        o, l, spread = defined(q, cache, tables, n, scale)
        # Rounding the result costs U, rounding the probabilities 2^-11 of sum p |v|, and those below 2^-14 at most 2^-25 each, where the largest
        # is 2^7 or more; all others in 32 bits: an exponent of at most 26 is off by 2^-19 at most, and sums of n terms.
        _, v64 = R.values(cache.cpu().numpy())
        rest = 2.0 ** -32 * np.abs(v64).sum((0, 1, 2)) / np.exp(l - nats)[..., None]
        tol = U[dtype] * np.abs(o) + (2.0 ** -11 + 2.0 ** -16) * spread + rest + 2.0 ** -24
        assert (np.abs(out - o) <= tol).all(), (nats, float((np.abs(out - o) / tol).max()))
        assert (np.abs(lse - l) <= 2.0 ** -19 * 26).all(), nats


@pytest.mark.parametrize("cut", [True, False], ids=["cut", "uncut"])
@pytest.mark.parametrize("form", FORMS)
def test_scales_and_queries_whose_product_leaves_the_range_of_32_bits(form, cut):
    n, rows, page = FORMS[form]
    g = torch.Generator().manual_seed(rows)
    k, v = torch.zeros(n, 64), torch.randn(n, 64, generator=g)
    k[:, 32:] = 2.0 ** -21 * torch.randint(1, 3, (n, 1), generator=g)
    cache, tables = cache_of(k, v, page)
    _, v64 = R.values(cache.cpu().numpy())
    v64 = v64.reshape(-1, 64)[:n]
    seen = np.arange(n)[None] <= n - rows + np.arange(rows)[:, None]

    def expect(q, scale, p, l):
        out, lse = attend(q, cache, tables, n, scale, cut)
        o = (p @ v64 / p.sum(1, keepdims=True))[:, None]
        tol = U[q.dtype] * np.abs(o) + 2.0 ** -10 * np.abs(v64).max()
        assert (np.abs(out - o) <= tol).all(), (scale, int(np.isnan(out).sum()))
        assert (np.abs(lse[:, 0] - l) <= 2.0 ** -16 * np.abs(l)).all(), scale
    # all scores 0 or next to it, with keys that the mask hides: the mean of the values that a row sees
    p = seen.astype(float)
    for dtype, size, scale in ((torch.bfloat16, 1e-38, 1e-10), (torch.bfloat16, 1e-39, 0.1), (torch.float16, 1.0, 1e-40), (torch.float16, 0.0, 1e30),
                               (torch.bfloat16, 0.0, 1e30)):
        expect(torch.full((rows, 1, 64), size).to(dtype).cuda(), scale, p, np.log(p.sum(1)))
    # queries next to 2^128 where the keys are 0: 0 as well, for any scale below 2^13
    q = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device="cuda")
    q[:, :, :32] = 1.5 * 2.0 ** 127
    for scale in (0.125, 1.9, 7.0, 5000.0, -5000.0):
        expect(q, scale, p, np.log(p.sum(1)))


def one_largest(q, cache, tables, n, scale):
    """Where each row's largest score is far above all others in 32 bits: the mean of the values of the keys that have it, and lse."""
    k, v = (x.reshape(-1, q.shape[-1])[:n] for x in R.values(cache.cpu().numpy()))
    rows = q.shape[0]
    x = f64(q)[:, 0] @ k.T * scale
    x[np.arange(n)[None] > n - rows + np.arange(rows)[:, None]] = -np.inf
    top = x.max(1, keepdims=True)
    p = (x == top).astype(float)
    second = np.where(p > 0, -np.inf, x).max(1)
    assert np.isfinite(top).all() and (top[:, 0] - second > 2.0 ** -8 * np.abs(top[:, 0])).all()
    return (p @ v / p.sum(1, keepdims=True))[:, None], top + np.log(p.sum(1, keepdims=True))


@pytest.mark.parametrize("cut", [True, False], ids=["cut", "uncut"])
@pytest.mark.parametrize("form", FORMS)
def test_scores_of_any_size(form, cut):
    """Scores from 1e5 to 1e37, of both signs, far beyond what neighbouring numbers in 32 bits can tell apart by less than 1."""
    n, rows, page = FORMS[form]
    g = torch.Generator().manual_seed(rows)
    for dtype, size, scale in ((torch.float16, 3.0, 1e4), (torch.float16, 2e3, 1.7), (torch.float16, 3e4, 1.3), (torch.float16, 3e4, -0.7),
                               (torch.bfloat16, 1e8, 0.125), (torch.bfloat16, 3e30, 1.9), (torch.bfloat16, 3e30, -1.1)):
        base = torch.randint(1, 7, (64,), generator=g) * 2.0 ** 12
        k = base[None] * torch.where(torch.arange(n) % 7 == 3, 1.0, 0.5)[:, None]
        k[-rows:] = 0                                              # every row sees the same of the other keys
        k[-rows:, 0] = base[0] * 0.75                              # one channel: the largest where the scale turns all scores
        v = torch.randn(n, 64, generator=g)
        cache, tables = cache_of(k, v, page)
        q = ((torch.rand(rows, 1, 64, generator=g) * 0.5 + 0.5) * size).to(dtype).cuda()
        out, lse = attend(q, cache, tables, n, scale, cut)
        o, l = one_largest(q, cache, tables, n, scale)
        tol = U[dtype] * np.abs(o) + 2.0 ** -10 * np.abs(f64(v)).max()
        assert (np.abs(out - o) <= tol).all(), (dtype, size, scale, float(np.nanmax(np.abs(out - o) / tol)), int(np.isnan(out).sum()))
        assert (np.abs(lse - l) <= 2.0 ** -16 * np.abs(l)).all(), (dtype, size, scale)
    # queries next to 2^127, where the keys are small
    k[-rows:] = 0
    cache, tables = cache_of(k * 2.0 ** -34, v, page)
    q = ((torch.rand(rows, 1, 64, generator=g) * 0.5 + 0.5) * 2.0 ** 127).bfloat16().cuda()
    for scale in (0.125, 7.0, 500.0):
        out, lse = attend(q, cache, tables, n, scale, cut)
        o, l = one_largest(q, cache, tables, n, scale)
        tol = U[q.dtype] * np.abs(o) + 2.0 ** -10 * np.abs(f64(v)).max()
        assert (np.abs(out - o) <= tol).all(), (scale, int(np.isnan(out).sum()))
        assert (np.abs(lse - l) <= 2.0 ** -16 * np.abs(l)).all(), scale
