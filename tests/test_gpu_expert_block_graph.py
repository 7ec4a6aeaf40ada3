"""The expert feed-forward block of the example, forward and backward, captured in a CUDA graph and
replayed on other rows and lengths."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import expert_encoder_layer as ex  # noqa: E402
import paper_2310_07109_gb300 as sc  # noqa: E402

pytestmark = pytest.mark.gpu


def test_the_block_in_a_graph():
    B, L, D, F, E, k = 3, 150, 128, 264, 8, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    bf = lambda *shape: torch.randn(shape, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    block = ex.ExpertFeedForward(D, F, E, k)
    ws = sc.new_expert_workspace(B, L, E, k, max(D, F))
    inputs = [(bf(B * L, D), bf(B * L, D), torch.tensor(rows, device="cuda").int())
              for rows in ([150, 20, 77], [1, 150, 0])]

    def both(H, dY, rows):
        Y, saved = block.forward(H, B, L, rows, ws)
        grads, dH = block.backward(dY, saved)
        live = (torch.arange(L, device="cuda")[None, :] < rows[:, None]).reshape(-1, 1)
        return [Y, torch.where(live, dH, 0)] + [grads[name] for name in sorted(grads)]

    right = [[t.clone() for t in both(*i)] for i in inputs]
    held = [t.clone() for t in inputs[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(*held)
    for i, r in zip(inputs[::-1], right[::-1]):
        for t, new in zip(held, i):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, r):
            assert torch.equal(a, b)
    assert sc.workspace_status(ws) == sc.SC_OK
