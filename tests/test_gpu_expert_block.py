"""The expert feed-forward block as a whole (examples/expert_encoder_layer.py) against a 64-bit
evaluation with autograd, behind the layer's attention half on ragged, pruned rows."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import expert_encoder_layer as ex  # noqa: E402

pytestmark = pytest.mark.gpu


def reference(block, H, rows, L, r, dY):
    """Y and every gradient in 64 bits, the choice of experts given."""
    live = (torch.arange(L, device="cuda")[None, :] < rows[:, None]).reshape(-1)
    p = {n: (block.half.get(n, v)).double().requires_grad_(True) for n, v in block.params.items()}
    h = H.double()[live].requires_grad_(True)
    logits = h @ p["W_r"][0].T
    expert = r["expert"][live].long()
    gate = torch.softmax(torch.gather(logits, 1, expert), dim=1)
    s = h
    for j in range(block.k):
        z = torch.zeros_like(h)
        for e in range(block.E):
            at = torch.nonzero(expert[:, j] == e)[:, 0]
            y = h[at] @ p["W_1"][e].T + p["b_1"][e]
            f = 0.5 * y * (1 + torch.erf(y / math.sqrt(2)))
            z = z.index_add(0, at, f @ p["W_2"][e].T + p["b_2"][e])
        s = s + gate[:, j: j + 1] * z
    Y = torch.nn.functional.layer_norm(s, (block.D,), p["gamma"], p["beta"], ex.EPS)
    names = list(p)
    grads = torch.autograd.grad(Y, [p[n] for n in names] + [h], dY.double()[live])
    return live, Y.detach(), dict(zip(names, grads[:-1])), grads[-1]


@pytest.mark.parametrize("B,L,D,F,E,k", [(3, 200, 256, 512, 8, 2), (1, 450, 128, 264, 16, 4)])
def test_block_against_64_bits(B, L, D, F, E, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(B + L)
    X = torch.randn(B, L, D, device="cuda", generator=g).to(torch.bfloat16)
    H, rows = ex.attention_half(X, ex.attention_weights(D), 32, 0.7)
    assert int(rows.min()) < L                       # something was pruned: the batch is ragged
    block = ex.ExpertFeedForward(D, F, E, k, seed=B)
    Y, saved = block.forward(H, B, L, rows)
    dY = torch.randn(B * L, D, device="cuda", generator=g).to(torch.bfloat16)
    grads, dH = block.backward(dY, saved)
    live, Yr, gr, dHr = reference(block, H, rows, L, saved["route"], dY)
    # stored in bf16 on the way: F, the value before GELU, Z, dZ, dpre, the slots' dH, the router's
    # dlogits; each rounds by 2^-9 of itself in the 2-norm, and at most six follow one another
    near = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    bound = 6 * 2.0 ** -9
    assert near(Y[live], Yr) <= bound
    assert near(dH[live], dHr) <= bound
    for name in gr:
        assert near(grads[name], gr[name]) <= bound, name
    assert bool((Y[~live] == 0).all())


def test_the_example_learns():
    losses = ex.main(B=2, L=256, D=256, F=512, E=8, k=2, steps=6, quiet=True)
    assert all(b < a for a, b in zip(losses, losses[1:]))
