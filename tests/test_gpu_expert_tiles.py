"""Products grouped by expert where each pair of SMs has several tiles of 64 to 256 slots:
what is kept from one tile to the next (values before GELU copied ahead, bias loaded ahead,
write-back areas used again, sums of several accumulators) against plain 64-bit products."""
import pytest

import test_gpu_expert as ops

pytestmark = pytest.mark.gpu

# 38 tiles of slots (33 to 256 in each), five or six of features: 190 to 228 for 76 pairs
COUNTS = [1500, 0, 257, 2100, 33, 900, 1300, 64, 1700, 511]


@pytest.mark.parametrize("N,K", [(1536, 1032), (1288, 1536)])
@pytest.mark.parametrize("gather,pad,gelu,pre,f32,bias,first", [
    (True, 0, True, True, False, True, 0),
    (False, 8, True, True, False, True, 3),
    (True, 16, True, False, False, True, 0),
    (False, 0, False, False, False, False, 0),
    (False, 0, True, True, True, True, 1),
    (True, 8, True, False, True, True, 0),
])
def test_forward_over_several_tiles(N, K, gather, pad, gelu, pre, f32, bias, first):
    ops.test_expert_linear_forward(COUNTS, N, K, gather, pad, gelu, pre, f32, bias, first)


@pytest.mark.parametrize("N,K", [(1032, 1536), (1536, 1288)])
@pytest.mark.parametrize("pad,pre,f32,first", [(0, True, False, 0), (8, False, False, 2), (16, True, True, 0),
                                               (0, False, True, 5)])
def test_backward_input_over_several_tiles(N, K, pad, pre, f32, first):
    ops.test_expert_linear_backward_input(COUNTS, N, K, pad, pre, f32, first)


@pytest.mark.parametrize("N,K", [(1536, 1032)])
@pytest.mark.parametrize("gather,pad,f32,bias,first", [(True, 0, True, True, 0), (False, 8, False, True, 3),
                                                       (True, 16, False, False, 0)])
def test_backward_weight_over_several_tiles(N, K, gather, pad, f32, bias, first):
    ops.test_expert_linear_backward_weight(COUNTS, N, K, gather, pad, f32, bias, first)
