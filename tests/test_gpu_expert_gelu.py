"""GELU and its slope in the expert products, over the whole range of their argument: the far
negative tail to its relative precision, and the limits.

The argument is exact: the forward product's rows are zero and the bias holds the arguments;
the gradient's product is 1 and the slope is read off it.  GELU is stated to be within
(16 + x^2) 2^-24 of itself, its slope of Phi(x) + |x| phi(x) (the exponential's argument is
rounded, hence x^2), down to 2^-122 (the exponential of smaller ones is taken for 0)."""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FLOOR = 2.0 ** -122


def phi_cdf(x):
    return 0.5 * torch.special.erfc(-x / math.sqrt(2))


def density(x):
    return torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def arguments(n):
    """n values in [-40, 40]: dense to 14, and to both sides of 0 over all its binades."""
    third = n // 3
    near = torch.logspace(-30, 0.6, third // 2, dtype=torch.float64)
    far = torch.linspace(14, 40, n - third - 2 * (third // 2), dtype=torch.float64)
    far[::2] *= -1
    return torch.cat([torch.linspace(-14, 14, third, dtype=torch.float64), near, -near, far]).float().cuda()


# (slots, experts, which kernel the sizes select)
KERNELS = [(4, 2, "few slots"), (40, 2, "few slots an expert"), (200, 1, "pairs of SMs")]


@pytest.mark.parametrize("M,E,_kernel", KERNELS)
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("pre", [True, False])
def test_gelu_over_its_range(M, E, _kernel, gather, f32, pre):
    N, K = 6000, 8
    x = arguments(E * N).view(E, N)
    X = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16)
    W = torch.ones(E, N, K, device="cuda", dtype=torch.bfloat16)
    off = torch.arange(E + 1, device="cuda").mul(M // E).int()
    token = torch.arange(M, device="cuda").int() if gather else None
    prev = torch.empty(M, N, device="cuda", dtype=torch.bfloat16) if pre else None
    got = sc.expert_linear_forward(X, W, off, token=token, bias=x, gelu=True, pre=prev, out_f32=f32).double()
    for e in range(E):
        v = x[e].double()
        ref = v * phi_cdf(v)
        rows = got[e * (M // E):(e + 1) * (M // E)]
        bound = ((16 + v * v) * U + (0 if f32 else 2.0 ** -8)) * ref.abs() * 1.01 + FLOOR
        bad = ~((rows - ref).abs() <= bound)
        assert not bool(bad.any()), "expert %d: %d off, at %s: %s, not %s" % (
            e, int(bad.sum()), v.expand_as(rows)[bad][:4].tolist(), rows[bad][:4].tolist(), ref.expand_as(rows)[bad][:4].tolist())
        if pre:
            assert torch.equal(prev[e * (M // E):(e + 1) * (M // E)], x[e].bfloat16().expand(M // E, N))


@pytest.mark.parametrize("M,E,_kernel", KERNELS)
@pytest.mark.parametrize("f32", [True, False])
def test_gelu_at_its_limits(M, E, _kernel, f32):
    N, K = 64, 8
    x = torch.randn(E, N, device="cuda")
    x[:, 0::8], x[:, 3::8], x[:, 4::8] = -math.inf, math.inf, math.nan   # each beside an ordinary value
    X = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16)
    W = torch.ones(E, N, K, device="cuda", dtype=torch.bfloat16)
    off = torch.arange(E + 1, device="cuda").mul(M // E).int()
    got = sc.expert_linear_forward(X, W, off, bias=x, gelu=True, out_f32=f32).double()
    for e in range(E):
        v = x[e].double()
        ref = torch.where(v == -math.inf, 0.0, v * phi_cdf(v))
        for row in got[e * (M // E):(e + 1) * (M // E)]:
            assert torch.equal(row.isnan(), v.isnan())
            assert bool((row[v == -math.inf] == 0).all()) and bool((row[v == math.inf] == math.inf).all())
            ok = v.isfinite()
            assert bool(((row - ref).abs()[ok] <= (2.0 ** -8 + 32 * U) * ref.abs()[ok]).all())


@pytest.mark.parametrize("M,E,_kernel", [(40, 2, "few slots an expert"), (200, 1, "pairs of SMs")])
@pytest.mark.parametrize("f32", [True, False])
def test_slope_over_its_range(M, E, _kernel, f32):
    N, K = 8, 8000
    bits = torch.arange(0, 0x4220, dtype=torch.int32)        # the bf16 values from 0 to 40
    every = torch.cat([bits, bits + 0x8000]).to(torch.uint16).view(torch.bfloat16)
    every = every[torch.randperm(len(every), generator=torch.Generator().manual_seed(2))].cuda()
    z = every.repeat(M * K // len(every) + 1)[:M * K].view(M, K).contiguous()
    dY = torch.zeros(M, N, device="cuda", dtype=torch.bfloat16)
    dY[:, 0] = 1
    W = torch.ones(E, N, K, device="cuda", dtype=torch.bfloat16)
    off = torch.arange(E + 1, device="cuda").mul(M // E).int()
    got = sc.expert_linear_backward_input(dY, W, off, pre=z, out_f32=f32).double()
    v = z.double()
    ref = phi_cdf(v) + v * density(v)
    bound = (16 + v * v) * U * (phi_cdf(v) + v.abs() * density(v)) + (0 if f32 else 2.0 ** -8) * ref.abs() * 1.01 + FLOOR
    bad = ~((got - ref).abs() <= bound)
    assert not bool(bad.any()), "%d off, at %s: %s, not %s" % (
        int(bad.sum()), v[bad][:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())
