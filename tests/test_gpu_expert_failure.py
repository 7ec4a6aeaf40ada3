"""The failure path of the expert products' bounded waits, on the GPU, without a fault: a wait of
every pair of CTAs runs out (the test hook), both CTAs abandon their work, await their
copies and products, and record the timeout; the next call on the same workspace is right."""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import expert as ex
import test_gpu_expert as ops

pytestmark = pytest.mark.gpu

STALL_NS = 200_000
COUNTS = [1500, 0, 257, 2100, 33, 900, 1300, 64]
N, K = 776, 1032


def forward(f32, gather, pre):
    g = ops.gen(5)
    X, token, M = ops.product_inputs(6, COUNTS, 301, K, gather=gather, pad=0)
    W = ops.bf16(ops.randn(g, len(COUNTS), N, K) / math.sqrt(K))
    z = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16) if pre else None
    out = torch.zeros(M, N, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    off = ops.offsets_of(COUNTS)

    def call(ws):
        sc.expert_linear_forward(X, W, off, token=token, gelu=pre, pre=z, out=out, workspace=ws)
        return [out] + ([z] if pre else [])
    return call


def backward_input(f32, pre):
    g = ops.gen(7)
    dY, _, M = ops.product_inputs(8, COUNTS, 0, N, gather=False, pad=0)
    W = ops.bf16(ops.randn(g, len(COUNTS), N, K) / math.sqrt(N))
    z = ops.bf16(ops.randn(g, M, K)) if pre else None
    out = torch.zeros(M, K, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    off = ops.offsets_of(COUNTS)

    def call(ws):
        sc.expert_linear_backward_input(dY, W, off, pre=z, out=out, workspace=ws)
        return [out]
    return call


def backward_weight(f32, gather, bias):
    X, token, M = ops.product_inputs(9, COUNTS, 301, K, gather=gather, pad=0)
    dY, _, _ = ops.product_inputs(10, COUNTS, 0, N, gather=False, pad=0)
    E = len(COUNTS)
    out = {"dW": torch.zeros(E, N, K, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)}
    if bias:
        out["dbias"] = torch.zeros(E, N, device="cuda")
    off = ops.offsets_of(COUNTS)

    def call(ws):
        sc.expert_linear_backward_weight(dY, X, off, token=token, out=out, workspace=ws)
        return list(out.values())
    return call


CALLS = {
    "forward": lambda: forward(False, False, False),
    "forward, gathered": lambda: forward(False, True, False),
    "forward, gathered, with pre": lambda: forward(False, True, True),
    "forward, fp32": lambda: forward(True, False, True),
    "forward, fp32, gathered": lambda: forward(True, True, True),
    "gradient of the rows": lambda: backward_input(False, False),
    "gradient of the rows, with pre": lambda: backward_input(False, True),
    "gradient of the rows, fp32": lambda: backward_input(True, True),
    "gradient of the weights": lambda: backward_weight(False, False, True),
    "gradient of the weights, no bias": lambda: backward_weight(False, False, False),
    "gradient of the weights, gathered": lambda: backward_weight(False, True, True),
    "gradient of the weights, fp32": lambda: backward_weight(True, False, True),
    "gradient of the weights, fp32, gathered": lambda: backward_weight(True, True, True),
}


@pytest.mark.parametrize("what", list(CALLS))
def test_expired_wait_is_reported_and_left_behind(what):
    call = CALLS[what]()
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    right = [t.clone() for t in call(ws)]
    assert sc.workspace_status(ws) == sc.SC_OK
    for _ in range(3):
        sc.debug_stall_waits(STALL_NS)
        try:
            began, ended = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            began.record()
            call(ws)
            ended.record()
        finally:
            sc.debug_stall_waits(0)
        assert sc.workspace_status(ws) == sc.SC_ERR_TIMEOUT
        assert sc.workspace_status(ws) == sc.SC_OK            # the query cleared the word
        # the other CTA of a pair does not wait its own two seconds
        assert began.elapsed_time(ended) < 500
        for a, b in zip(call(ws), right):
            assert torch.equal(a, b)
        assert sc.workspace_status(ws) == sc.SC_OK


def test_status_of_calls_without_a_workspace():
    """Reported too, whichever stream the call was on, until it is asked for."""
    calls = [CALLS[what]() for what in ("forward", "gradient of the rows", "gradient of the weights")]
    right = [[t.clone() for t in call(None)] for call in calls]
    assert sc.expert_status() == sc.SC_OK
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side):
        for i, call in enumerate(calls):
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                sc.debug_stall_waits(STALL_NS)
                try:
                    call(None)
                finally:
                    sc.debug_stall_waits(0)
                got = [t.clone() for t in call(None)]   # (a later call does not clear it)
            torch.cuda.synchronize()
            assert sc.expert_status() == sc.SC_ERR_TIMEOUT
            assert sc.expert_status() == sc.SC_OK
            for a, b in zip(got, right[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("first", [False, True])   # the first call without a workspace at all?
def test_calls_without_a_workspace_in_a_graph(first, monkeypatch):
    call = CALLS["forward"]()
    right = [t.clone() for t in call(None)]
    if first:
        monkeypatch.setattr(ex, "_products", {})
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        out = call(None)
    for t in out:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, right):
        assert torch.equal(a, b)
    assert sc.expert_status() == sc.SC_OK
