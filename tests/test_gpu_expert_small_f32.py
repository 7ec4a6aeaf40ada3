"""fp32 products of few slots an expert are as near as fp32 sums get.

The tensor cores' additions cut off, up to a unit in the last place (0.36 2^-23 of the sum on
average over a binade).  In the sum of a stage of 64 products there are four, after 16, 32,
48 and 64 of them: of normal products these partial sums are (4 + 5.7 + 6.9 + 8) / 8 of the
stage's sum together, 1.1 2^-23 of it are cut off, and the stages' signs are independent.
Adding n stages rounds off 0.72 2^-24 sqrt(n / 6) of the result (2-norm).  Half as much again
is allowed."""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("depth", [256, 520, 2048, 8192])
def test_fp32_products_of_few_slots(backward, depth):
    E, each, width = 2, 40, 512
    g = torch.Generator(device="cuda")
    g.manual_seed(depth)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    rows, W = randn(E * each, depth), randn(*((E, depth, width) if backward else (E, width, depth)))
    off = torch.tensor([0, each, 2 * each], device="cuda").int()
    got = (sc.expert_linear_backward_input if backward else sc.expert_linear_forward)(rows, W, off, out_f32=True).double()
    ref = torch.cat([rows[e * each:(e + 1) * each].double() @ (W[e].double() if backward else W[e].double().T)
                     for e in range(E)])
    off_by = float((got - ref).norm() / ref.norm())
    bound = 1.5 * math.hypot(1.1 * 2.0 ** -23, 0.72 * 2.0 ** -24 * math.sqrt(depth / 64 / 6))
    assert off_by <= bound, "%.3g against %.3g" % (off_by, bound)
