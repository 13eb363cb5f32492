"""Scratch memory in graphs that torch records, and in graphs that the program records itself (hipStreamBeginCapture)."""
import ctypes

import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import f64, reference, setup
from tests.test_gpu_rope import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hip():
    torch.cuda.init()
    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64.so" in line)   # the one that torch uses
    return ctypes.CDLL(path)


def record(hip, call):
    """What `call` enqueues on torch's current stream as a graph of the runtime's own: (the number of its nodes, replay)."""
    graph, exe, n, vp = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_size_t(), ctypes.c_void_p
    stream = vp(torch.cuda.current_stream().cuda_stream)
    assert hip.hipStreamBeginCapture(stream, 2) == 0               # 2: hipStreamCaptureModeRelaxed
    try:
        call()
    finally:
        assert hip.hipStreamEndCapture(stream, ctypes.byref(graph)) == 0
    assert hip.hipGraphGetNodes(graph, None, ctypes.byref(n)) == 0
    if n.value:
        assert hip.hipGraphInstantiate(ctypes.byref(exe), graph, None, None, ctypes.c_size_t(0)) == 0

    def replay():
        assert hip.hipGraphLaunch(exe, stream) == 0
        torch.cuda.synchronize()
    return n.value, replay


@pytest.mark.parametrize("plain", [True, False], ids=["native", "python"])
def test_attention_in_a_recording_of_the_program(hip, plain):
    """Without a workspace the keys are not cut, so one kernel and no memory of torch's; with one, two kernels."""
    from paper_2403_16863_amd import kv4
    s = setup(([5000, 30], [1, 1], 8, 2, 128, 16, True), torch.float16)
    want = reference(s)
    number = int if plain else np.int64                            # a count that only the Python path takes
    need = kv4.kv4_attn_workspace(2, 2, 8, 2, 128, 16, s["tables"].shape[1], 1)
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    given = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(workspace=None):
        kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], out, lse, True, s["scale"], s["cu"], number(1), workspace)
    call()                                                         # torch holds memory of that size from here on
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        for workspace, kernels in ((None, 1), (given, 2)):
            nodes, replay = record(hip, lambda: call(workspace))
            assert nodes == kernels
            others = torch.full((need,), 77, dtype=torch.uint8, device="cuda")
            for _ in range(3):
                out.fill_(float("nan"))
                lse.fill_(float("nan"))
                replay()
                assert np.abs(f64(out) - want[0]).max() <= 2.0 ** -9 * want[2].max() and np.abs(f64(lse) - want[1]).max() < 1e-3
                assert bool((others == 77).all())
    torch.cuda.synchronize()


def test_backward_in_a_recording_of_the_program(hip):
    """Refused without a workspace; with one the same as eager."""
    from paper_2403_16863_amd import rope
    B, N, H, Hkv, d = 1, 600, 4, 2, 64
    q, k, dqo, dko, (qw, kw), c, s, positions = inputs(B, N, H, Hkv, d, torch.float16, torch.float16)
    outs = [torch.empty(B, N, n, d, dtype=torch.float16, device="cuda") for n in (H, Hkv)] + [torch.empty(d, device="cuda") for _ in range(2)]

    def call(**more):
        rope.qk_norm_rope_bwd(dqo, dko, q, k, outs[0], outs[1], c, s, positions, qw, kw, outs[2], outs[3], **more)
    call()
    want = [t.clone() for t in outs]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        def refused():
            with pytest.raises(ValueError, match="recording"):
                call()
        assert record(hip, refused)[0] == 0
        space = torch.empty(rope.qk_norm_rope_bwd_workspace(B, N, H, Hkv, d), dtype=torch.uint8, device="cuda")
        nodes, replay = record(hip, lambda: call(workspace=space))
        assert nodes == 2
        for _ in range(3):
            for t in outs:
                t.fill_(float("nan"))
            replay()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
    torch.cuda.synchronize()


@pytest.mark.parametrize("pool", ["own", "handle"])
@pytest.mark.parametrize("plain", [True, False], ids=["native", "python"])
def test_attention_in_a_graph_of_torch_is_cut_as_it_is_without(plain, pool):
    from paper_2403_16863_amd import kv4
    s = setup(([5000, 30], [1, 1], 8, 2, 128, 16, True), torch.float16)
    number = int if plain else np.int64
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")

    def call():
        kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], out, lse, True, s["scale"], s["cu"], number(1))
    call()
    want = out.clone(), lse.clone()
    uncut = torch.cuda.Stream()
    uncut.wait_stream(torch.cuda.current_stream())
    o, l = torch.empty_like(out), torch.empty_like(lse)
    torch.cuda.synchronize()
    kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], o, l, True, s["scale"], s["cu"], 1, stream=uncut.cuda_stream)
    torch.cuda.synchronize()
    assert not torch.equal(l, want[1])                             # the two differ in their last bits
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, pool=torch.cuda.graph_pool_handle() if pool == "handle" else None):
        call()
    for _ in range(3):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("which", ["own", "default"])
def test_calls_beside_a_recording_of_torch_in_another_thread(which):
    """They take memory of their own streams, and end neither the recording nor themselves."""
    import threading

    from paper_2403_16863_amd import kv4, rope
    s = setup(([5000, 30], [1, 1], 8, 2, 128, 16, True), torch.float16)
    out, lse = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda")
    q, _, dqo, _, (qw, _), c, sn, positions = inputs(1, 600, 4, 2, 64, torch.float16, torch.float16)
    dq, dw = torch.empty(1, 600, 4, 64, dtype=torch.float16, device="cuda"), torch.empty(64, device="cuda")

    def calls():
        kv4.kv4_attn(s["q"], s["cache"], s["tables"], s["lens"], out, lse, True, s["scale"], s["cu"], 1)
        rope.qk_norm_rope_bwd(dqo, None, q, None, dq, None, c, sn, positions, qw, None, dw, None)
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, lse, dq, dw)]
    for t in (out, lse, dq, dw):
        t.zero_()
    errors = []

    def beside():
        try:
            with torch.cuda.stream(torch.cuda.Stream() if which == "own" else torch.cuda.default_stream()):
                calls()
        except Exception as e:
            errors.append(e)
    x, y = torch.arange(8.0, device="cuda"), torch.zeros(8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        torch.add(x, 1, out=y)
        thread = threading.Thread(target=beside)
        thread.start()
        thread.join()
        y.mul_(2)
    assert not errors
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, lse, dq, dw), want))
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, 2 * (x + 1))
