"""The weight gradient where an expert has very many slots: its sums do not lose with their length."""
import pytest
import torch

import paper_2310_07109_gb300 as sc
import test_gpu_expert as ops

pytestmark = pytest.mark.gpu


def bf16_ulp(x):
    """The distance of neighbouring bf16 values at x (x not 0)."""
    return torch.exp2(torch.floor(torch.log2(x.abs())) - 7)


@pytest.mark.parametrize("gather", [True, False])
def test_bf16_weight_gradient_of_millions_of_slots(gather):
    """Positive products, so that what each addition cuts off adds up.  Sums of 512 products are
    cut off by at most 32 units in the last place (2^-18), their sum in fp32 is rounded 8192
    times, half a unit of 2^-23 at most and either way: 2^-10 of the result at the very most,
    an eighth of bf16's unit beside the rounding's half."""
    counts, N, K = [1000, 1 << 22, 0, 77], 24, 16
    g = ops.gen(3)
    M = sum(counts)
    x_rows = 5000 if gather else M
    X = ops.bf16(torch.rand((x_rows, K), device="cuda", generator=g) + 0.5)
    dY = ops.bf16(torch.rand((M, N), device="cuda", generator=g) + 0.5)
    token = torch.randint(0, x_rows, (M,), device="cuda", generator=g).int() if gather else None
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    got = sc.expert_linear_backward_weight(dY, X, ops.offsets_of(counts), token=token, out_f32=False, workspace=ws)
    assert sc.workspace_status(ws) == 0
    lo = 0
    for e, c in enumerate(counts):
        rows = (X[lo:lo + c] if token is None else X[token[lo:lo + c].long()]).double()
        ref = dY[lo:lo + c].double().T @ rows
        off = (got["dW"][e].double() - ref).abs()
        if c == 0:
            assert bool((off == 0).all())
        else:
            assert bool((off <= (0.5 + 0.125) * bf16_ulp(ref)).all()), "expert %d: %.3g units off" % (
                e, float((off / bf16_ulp(ref)).max()))
        lo += c


@pytest.mark.parametrize("counts,N,K", [
    ([70000], 264, 520),                              # three column blocks and two of features, the last ones partial
    ([9, 30000, 0, 1, 20000, 63, 16000], 136, 776),
    ([0, 66000, 0], 8, 8),
    ([700] * 100, 200, 72),
])
@pytest.mark.parametrize("gather,pad,bias", [(True, 0, True), (False, 8, True), (True, 16, False)])
def test_bf16_weight_gradient_in_spans(counts, N, K, gather, pad, bias):
    ops.test_expert_linear_backward_weight(counts, N, K, gather, pad, False, bias, 3)


@pytest.mark.parametrize("c", [1, 64, 65, 4096, 4200, 1 << 16])
def test_bias_gradient_beside_a_large_value(c):
    """A slot of 2^24 and ones: additions of single values to the sum so far would lose every one.
    16 slots, 64 such sums and one more for each 4096 slots are added in turn, then four warps' sums."""
    M, N, K = c + 3, 40, 8
    dY = torch.ones(M, N, device="cuda", dtype=torch.bfloat16)
    dY[0] = 2.0 ** 24
    X = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16)
    got = sc.expert_linear_backward_weight(dY, X, ops.offsets_of([c, 0, 3]))["dbias"].double()
    bound = (16 + 64 + c / 4096 + 4) * 2.0 ** -24 * (2.0 ** 24 + c - 1)
    assert bool(((got[0] - (2.0 ** 24 + c - 1)).abs() <= bound).all()), "%g off" % float(2.0 ** 24 + c - 1 - got[0].min())
    assert bool((got[1] == 0).all()) and bool((got[2] == 3).all())
