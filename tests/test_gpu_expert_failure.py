"""The failure path of the expert products' bounded waits, on the GPU, without a fault: a wait of
every pair of CTAs runs out (the test hook), both CTAs abandon their work, await their
copies and products, and record the timeout; the next call on the same workspace is right."""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc
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

    def call(ws):
        sc.expert_linear_forward(X, W, ops.offsets_of(COUNTS), token=token, gelu=pre, pre=z, out=out, workspace=ws)
        return [out] + ([z] if pre else [])
    return call


def backward_input(f32, pre):
    g = ops.gen(7)
    dY, _, M = ops.product_inputs(8, COUNTS, 0, N, gather=False, pad=0)
    W = ops.bf16(ops.randn(g, len(COUNTS), N, K) / math.sqrt(N))
    z = ops.bf16(ops.randn(g, M, K)) if pre else None
    out = torch.zeros(M, K, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)

    def call(ws):
        sc.expert_linear_backward_input(dY, W, ops.offsets_of(COUNTS), pre=z, out=out, workspace=ws)
        return [out]
    return call


def backward_weight(f32, gather, bias):
    X, token, M = ops.product_inputs(9, COUNTS, 301, K, gather=gather, pad=0)
    dY, _, _ = ops.product_inputs(10, COUNTS, 0, N, gather=False, pad=0)
    E = len(COUNTS)
    out = {"dW": torch.zeros(E, N, K, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)}
    if bias:
        out["dbias"] = torch.zeros(E, N, device="cuda")

    def call(ws):
        sc.expert_linear_backward_weight(dY, X, ops.offsets_of(COUNTS), token=token, out=out, workspace=ws)
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
