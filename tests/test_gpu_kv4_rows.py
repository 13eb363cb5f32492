"""Rows of the cached attention that belong to no sequence, uncut calls on other streams, and the norms' backward pass over more tokens than
one round of its workgroups takes."""
import numpy as np
import pytest
import torch

from tests import kv4_ref as R
from tests.test_gpu_kv4 import CASES, DTYPES, check, f64, random_case, reference, run, setup
from tests.test_gpu_rope import angles, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,most,most_q,d", [(3, 5000, 1, 64), (5, 3000, 9, 128), (4, 2600, 40, 64), (3, 2300, 600, 64), (64, 2300, 1, 128), (70, 2200, 3, 64)])
def test_rows_of_nobody_beside_cut_sequences(B, most, most_q, d, dtype):
    """Rows before the first sequence, behind the last, and beyond max_q stay as they are, whatever lies in the scratch memory."""
    from paper_2403_16863_amd import kv4
    s = setup(random_case(B, most, most_q, 4, 2, d, B), dtype, seed=B)
    want = reference(s)
    rows = s["q"].shape[0]
    pad = torch.zeros(7, 4, d, dtype=dtype, device="cuda")
    s["q"], s["cu"] = torch.cat((pad, s["q"], pad)), s["cu"] + 7
    need = kv4.kv4_attn_workspace(rows + 14, B, 4, 2, d, 16, s["tables"].shape[1], s["max_q"])
    assert need > 0
    space = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    out, lse = run(s, workspace=space)
    check(out[7:-7], lse[7:-7], want, dtype, scores=60)
    for x in (out, lse):
        assert torch.isnan(x[:7]).all() and torch.isnan(x[-7:]).all()
    if s["max_q"] > 2:
        # Sequences with more queries than max_q says: the first of them are computed, causal from the sequence's end with that number.
        less, cu = s["max_q"] - 2, s["cu"].tolist()
        s["max_q"] = less
        space.fill_(255)
        out, lse = run(s, workspace=space)
        for b in range(B):
            assert torch.isnan(lse[cu[b] + less:cu[b + 1]]).all() and torch.isnan(out[cu[b] + less:cu[b + 1]]).all()
            assert not torch.isnan(lse[cu[b]:min(cu[b] + less, cu[b + 1])]).any()
        assert torch.isnan(lse[:7]).all() and torch.isnan(lse[-7:]).all()


def uncut(s):
    """On a stream that torch does not know as current no memory is taken; it waits for the fill of the outputs."""
    out, lse = torch.full_like(s["q"], float("nan")), torch.full(s["q"].shape[:2], float("nan"), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(s, stream=side.cuda_stream, out=out, lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES + [([3000, 40, 0, 2500], [300, 30, 5, 256], 8, 2, 64, 16, True), ([4100], [1], 4, 1, 128, 16, True),
                                          ([2600, 2100], [16, 30], 2, 1, 64, 16, True)], ids=lambda c: "x".join(map(str, c[0])))
def test_uncut_calls_match_the_definition(case, dtype):
    s = setup(case, dtype)
    check(*uncut(s), reference(s), dtype, scores=60)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,N,H,Hkv,d,interleaved", [(1, 40003, 2, 1, 64, False), (3, 11001, 1, 2, 128, True)])
def test_backward_over_many_rounds_of_tokens(B, N, H, Hkv, d, interleaved, dtype):
    from paper_2403_16863_amd import rope
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, dtype, torch.float32)
    eps = 1e-5
    dq, dk = (torch.full((B, N, n, d), float("nan"), dtype=dtype, device="cuda") for n in (H, Hkv))
    dqw, dkw = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    rope.qk_norm_rope_bwd(dqo, dko, q, k, dq, dk, c, s, positions, qw, kw, dqw, dkw, eps, interleaved)
    co, si = angles(c, s, positions)
    for x, w, dy, dx, dw in ((q, qw, dqo, dq, dqw), (k, kw, dko, dk, dkw)):
        x64, dy64 = f64(x), f64(dy)
        gx, gw = R.norm_rope_bwd(dy64, x64, f64(w), co, si, eps, interleaved)
        size = np.abs(gx).max(-1, keepdims=True) + np.abs(dy64).max(-1, keepdims=True)
        unit = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
        assert (np.abs(f64(dx) - gx) <= unit * np.abs(gx) + 2.0 ** -18 * size * (1 + np.abs(x64).max())).all()
        # Each term g r x has about 12 roundings in 32 bits (the turn, the norm, the product), of sizes of both of a pair's gradients; a sum runs through
        # fewer than 64 additions: a lane's own, those of a column in the workgroup, and 16 of 128 threads with the tree above them.
        r = 1 / np.sqrt((x64 * x64).mean(-1, keepdims=True) + eps)
        pair = np.abs(R.rotate(np.abs(dy64), np.abs(co), -np.abs(si), interleaved, turn=-1)) + np.abs(R.rotate(np.abs(dy64), np.abs(co), np.abs(si), interleaved, turn=-1))
        terms = (pair * np.abs(x64) * r).reshape(-1, d).sum(0)
        assert (np.abs(f64(dw) - gw) <= (12 + 64) * 2.0 ** -24 * terms).all(), float((np.abs(f64(dw) - gw) / terms).max() * 2 ** 24)
