"""Eviction where the cut lies among the largest weights there are (+inf, the largest float) and the list has negative ones
too: the range of keys is then wider than 2^31 and its last part ends at the end of the 32 bits.  Against the plain
ranking of ``cache_reference``, bit for bit."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu

INF, BIG = math.inf, torch.finfo(torch.float32).max


def make(lists, C, lens, accs, seed):
    """One sequence a list, one key head of 16 features whose values name their slot; accs: of each list's slots in use."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    K = torch.randn(lists, 1, C, 16, device="cuda", generator=g).to(torch.bfloat16)
    V = torch.randn(lists, 1, C, 16, device="cuda", generator=g).to(torch.bfloat16)
    acc = torch.zeros(lists, 1, C, device="cuda")
    pos = torch.zeros(lists, 1, C, dtype=torch.int32, device="cuda")
    for b, (n, a) in enumerate(zip(lens, accs)):
        acc[b, 0, :n] = a[torch.randperm(n, device="cuda", generator=g)]
        pos[b, 0, :n] = 10 + torch.randperm(n, device="cuda", generator=g).int()
    return dict(K=K, V=V, acc=acc, pos=pos, len=torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None],
                seen=torch.tensor([n + 10 for n in lens], dtype=torch.int32, device="cuda"))


def check(cache, budget, sinks=0, recent=0):
    K, V, acc, pos, length = ref.evict(cache, budget, 0, sinks, recent)
    B, G, C = acc.shape
    # the workspace's plans lie between others' bytes, which stay
    size = sc.cache_workspace_size(B, C, 1, 1, width=16)
    raw = torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda")
    at = -raw.data_ptr() % 256
    ws = raw[at:at + size]
    ws.zero_()
    out = dict(acc=torch.full_like(acc, 9), pos=torch.full_like(pos, 9), len=torch.zeros_like(length))
    sc.cache_evict(cache, budget=budget, sinks=sinks, recent=recent, out=out, workspace=ws)
    live = torch.arange(C, device="cuda") < length[..., None]
    assert torch.equal(out["len"], length)
    assert torch.equal(out["pos"][live], pos[live]) and torch.equal(out["acc"][live], acc[live])
    assert torch.equal(cache["K"], K) and torch.equal(cache["V"], V)
    assert bool((raw[:at] == 77).all()) and bool((raw[at + size:] == 77).all())


def column(n, top, low, ordinary):
    """n weights: top's values in equal shares at the front, then one of each of `low`, then ordinary ones."""
    a = ordinary.clone()
    a[:len(top)] = torch.tensor(top)
    a[len(top):len(top) + len(low)] = torch.tensor(low)
    return a.cuda()


@pytest.mark.parametrize("n,C", [(8, 8), (300, 303), (9000, 9000), (20001, 20001), (50003, 50003)])   # 1, 1, 2, 4 and 8 CTAs a list
@pytest.mark.parametrize("low", [(-INF,), (-1.0,), (-INF, -BIG, -1.0, -0.0)])
@pytest.mark.parametrize("kind", ["inf", "big", "both", "from 2^127"])
def test_the_cut_among_the_largest(n, C, low, kind):
    g = torch.Generator()
    g.manual_seed(n)
    k = max(2, n // 3)
    for many in (k - 1, k, k + 1):   # largest ones for a budget of k: the cut beyond them, at their end, inside
        top = {"inf": [INF] * many, "big": [BIG] * many, "both": [INF, BIG] * (many // 2) + [INF] * (many % 2),
               "from 2^127": [2.0 ** 127 * (1 + i / (many + 1)) for i in range(many)]}[kind]
        a = column(n, top, low[:n - many], torch.rand(n, generator=g))
        ordinary = torch.rand(n, generator=g).cuda()
        check(make(2, C, [n, n], [a, ordinary], n + many), k)   # and the list behind it, an ordinary one


@pytest.mark.parametrize("n", [8, 9000, 20001, 50003])
def test_nothing_but_infinities(n):
    """Half of the slots given up with -inf, half held with +inf, budgets on both sides and at the border; ties all over."""
    half = n // 2
    a = torch.full((n,), -INF)
    a[:half] = INF
    for k in (half - 1, half, half + 1, n - 1):
        check(make(2, n, [n, n], [a.cuda(), a.cuda()], k), k)


@pytest.mark.parametrize("n", [40, 9000, 50003])
def test_held_by_position_and_by_weight(n):
    """Protected positions, then +inf, then the largest float: the cut within the last of them."""
    a = torch.rand(n) - 0.5
    a[:n // 4], a[n // 4:n // 2] = INF, BIG
    check(make(2, n, [n, n - 3], [a.cuda(), a[:n - 3].cuda()], n), n // 3 + n // 8, sinks=n // 40 + 10, recent=n // 16)
