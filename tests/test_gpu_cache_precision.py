"""What is left of the softmax's weights where they meet V: as two 16-bit values a weight loses some u^2 of itself in place of u (u:
half a step of the type), so O is the 64-bit result rounded once, but for the errors of 32-bit scores and sums.

Tolerance of O, size = P |V|:  u |O| for the one rounding;  4 u^2 size for the weights: the second value is at most 2 u + u of the
weight and is rounded to u of itself, which is 3 u^2;  scores of d products in 32 bits are within (d + 16) 2^-23 of their magnitudes, a weight within twice that,
2^-20 for the exponentials;  n 2^-23 size for the sums over n slots;  2^-25, half of fp16's smallest step, once for O and
2^-12 (the weights' scale) of it for each slot's second value."""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def inputs(T, H, Hk, d, n, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    cache = dict(K=randn(1, Hk, n, d).to(dtype), V=randn(1, Hk, n, d).to(dtype), acc=torch.zeros(1, 1, n, device="cuda"),
                 pos=torch.randperm(n, device="cuda", generator=g).int()[None, None].contiguous(),
                 len=torch.full((1, 1), n, dtype=torch.int32, device="cuda"), seen=torch.full((1,), n, dtype=torch.int32, device="cuda"))
    return cache, randn(T, H * d).to(dtype)


def weights(cache, Q, T):
    """P [H, T, n] in 64 bits, and the scores' magnitudes."""
    Hk, n, d = cache["K"].shape[1:]
    H = Q.shape[1] // d
    k = cache["K"][0].double().repeat_interleave(H // Hk, 0)
    q = Q.double().view(T, H, d).transpose(0, 1)
    at = int(cache["seen"]) - T + torch.arange(T, device="cuda")
    s = torch.where(cache["pos"][0, 0] <= at[:, None], q @ k.transpose(1, 2) / math.sqrt(d), -math.inf)
    return torch.softmax(s, 2), float((q.abs() @ k.abs().transpose(1, 2)).max()) / math.sqrt(d)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n", [3, 20, 90, 700])
@pytest.mark.parametrize("T,H,Hk,d", [(1, 12, 12, 64), (1, 16, 2, 128), (2, 16, 2, 64), (3, 8, 1, 128), (2, 20, 2, 64), (3, 10, 5, 128), (90, 4, 4, 64),
                                      (90, 4, 2, 128)])
def test_weights_keep_their_digits(T, H, Hk, d, n, dtype):
    """Up to 16, up to 32 and more rows a key head; features whose terms cancel show what the weights lost."""
    T = min(T, n)
    cache, Q = inputs(T, H, Hk, d, n, dtype, n + T)
    P, most = weights(cache, Q, T)
    v = cache["V"][0].double().repeat_interleave(H // Hk, 0)
    want, size = (P @ v).transpose(0, 1).reshape(T, H * d), (P @ v.abs()).transpose(0, 1).reshape(T, H * d)
    u = torch.finfo(dtype).eps / 2
    off = size * (4 * u * u + 2 * most * (d + 16) * 2.0 ** -23 + 2.0 ** -20 + n * 2.0 ** -23) + 2.0 ** -25 * (1 + 2.0 ** -12 * n * float(v.abs().max()))
    got = sc.cache_attend(cache, Q, T=T)["O"].double()
    wrong = (got - want).abs() > want.abs() * u * 1.01 + off
    assert not bool(wrong.any()), "%d of %d off, worst %.3g for %.3g" % (
        int(wrong.sum()), wrong.numel(), float((got - want).abs()[wrong].max()), float(off.min()))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,H,Hk,d", [(1, 8, 2, 64), (1, 4, 4, 128), (5, 8, 2, 64), (5, 5, 1, 128), (40, 2, 1, 64), (40, 2, 2, 128)])
def test_infinities_of_v_stay_infinities(T, H, Hk, d, dtype):
    """A slot that every row sees has infinities in some features: those of O are infinite, the others as without it."""
    n = 150
    cache, Q = inputs(T, H, Hk, d, n, dtype, T)
    c = int(torch.nonzero(cache["pos"][0, 0] == 7)[0])
    plain = sc.cache_attend(cache, Q, T=T, out=dict(acc=torch.zeros_like(cache["acc"])))["O"].clone()
    cache["V"][0, :, c, 3], cache["V"][0, :, c, d - 1] = math.inf, -math.inf
    got = sc.cache_attend(cache, Q, T=T)["O"].view(T, H, d)
    assert bool((got[..., 3] == math.inf).all()) and bool((got[..., d - 1] == -math.inf).all())
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[3] = rest[d - 1] = False
    assert torch.equal(got[..., rest], plain.view(T, H, d)[..., rest])
