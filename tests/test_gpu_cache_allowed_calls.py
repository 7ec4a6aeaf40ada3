"""Calls that the header allows and that are easily missed: outputs in the place of inputs, some of the outputs apart from the
cache and some not, the most heads, no rows in use at all, caches of one slot."""
import itertools
import math

import pytest
import torch

import cache_reference as ref
import paper_2310_07109_gb300 as sc
from test_gpu_cache import check_attend, check_evict, copy, gen, i32, make_cache, randn, same

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def projection(g, T, H, Hk, d, dtype=BF):
    """Queries, keys and values as slices of one matrix."""
    qkv = randn(g, T, (H + 2 * Hk) * d).to(dtype)
    return qkv, qkv[:, :H * d], qkv[:, H * d:(H + Hk) * d], qkv[:, (H + Hk) * d:]


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,d,rot", [(3, 50, 6, 2, 64, 64), (1, 1, 12, 12, 64, 32), (2, 600, 4, 1, 128, 128), (1, 70, 3, 3, 80, 48)])
def test_rotation_and_gradient_in_place(B, L, H, Hk, d, rot, inter):
    g = gen(L + d)
    qkv, Q, K, V = projection(g, B * L, H, Hk, d)
    kw = dict(width=d, B=B, L=L, freq=sc.rotary_frequencies(rot)[0], interleaved=inter, gamma_q=1 + 0.2 * randn(g, d), gamma_k=1 + 0.2 * randn(g, d))
    before = qkv.clone()
    want = sc.rotate_forward(Q, K, **kw)
    dqkv, dQ, dK, _ = projection(g, B * L, H, Hk, d)
    dbefore = dqkv.clone()
    grads = sc.rotate_backward(dQ, dK, Q, K, **kw)
    got = sc.rotate_backward(dQ, dK, Q, K, out=dict(dQ=dQ, dK=dK), **kw)
    assert all(torch.equal(got[n], grads[n]) for n in grads)
    assert torch.equal(dqkv[:, (H + Hk) * d:], dbefore[:, (H + Hk) * d:]) and torch.equal(qkv, before)
    sc.rotate_forward(Q, K, out=dict(Q=Q, K=K), **kw)
    assert torch.equal(Q, want["Q"]) and torch.equal(K, want["K"]) and torch.equal(V, before[:, (H + Hk) * d:])


@pytest.mark.parametrize("B,L,H,Hk,d", [(3, 1, 8, 2, 64), (2, 200, 6, 3, 128)])
def test_append_with_queries_in_place(B, L, H, Hk, d):
    g = gen(L)
    cache = make_cache(g, B, Hk, 300, d, 1, [7 * (b + 1) for b in range(B)])
    qkv, Q, K, V = projection(g, B * L, H, Hk, d)
    kw = dict(L=L, freq=sc.rotary_frequencies(d)[0], gamma_q=1 + 0.2 * randn(g, d))
    other = copy(cache)
    want = sc.cache_append(other, Q, K, V, **kw)["Q"].clone()
    assert sc.cache_append(cache, Q, K, V, out={"Q": Q}, **kw)["Q"] is Q
    assert torch.equal(Q, want) and all(same(cache[n], other[n]) for n in cache)


@pytest.mark.parametrize("apart", [c for n in range(4) for c in itertools.combinations(("acc", "pos", "len"), n)])
@pytest.mark.parametrize("C,lens,budget", [(400, [400, 90, 120], 100), (1500, [1500, 1400, 3], 1200), (9100, [9100, 9000, 40], 5000), (50, [50, 20, 0], 60)])
def test_evict_with_some_outputs_apart(apart, C, lens, budget):
    g = gen(C)
    cache = make_cache(g, 3, 2, C, 64, 1, lens)
    K, V, acc, pos, length = ref.evict(cache, budget, 0, 2, 9)
    mine = copy(cache)
    out = {n: torch.full_like(mine[n], 9) for n in apart}
    got = sc.cache_evict(mine, budget=budget, sinks=2, recent=9, out=out)
    live = torch.arange(C, device="cuda") < length[..., None]
    assert same(mine["K"], K) and same(mine["V"], V) and torch.equal(got["len"], length)
    for n, want in (("acc", acc), ("pos", pos)):
        assert same(got[n][live], want[live]), n
        # behind the lists: as it was, apart from the cache and in it
        assert bool((got[n][~live] == 9).all()) if n in apart else same(got[n][~live], cache[n][~live]), n
    for n in apart + ("seen",):
        assert same(mine[n], cache[n]), n


@pytest.mark.parametrize("H,Hk,d,inter", [(1000, 24, 16, False), (512, 512, 16, True), (1, 1023, 32, False), (200, 56, 256, True)])
def test_the_most_heads(H, Hk, d, inter):
    """Rotation and its gradient of one part of the heads are those of that part alone."""
    g = gen(H)
    L = 5
    _, Q, K, _ = projection(g, L, H, Hk, d)
    dQ, dK = randn(g, L, H * d).to(BF), randn(g, L, Hk * d).to(BF)
    kw = dict(B=1, L=L, width=d, freq=sc.rotary_frequencies(d)[0], interleaved=inter, gamma_q=1 + 0.2 * randn(g, d), gamma_k=1 + 0.2 * randn(g, d))
    out, back = sc.rotate_forward(Q, K, **kw), sc.rotate_backward(dQ, dK, Q, K, **kw)
    total = {"Q": torch.zeros(d, dtype=torch.float64, device="cuda"), "K": torch.zeros(d, dtype=torch.float64, device="cuda")}
    part = 97
    for n, x, dy in (("Q", Q, dQ), ("K", K, dK)):
        kw1 = dict(kw, gamma_q=kw["gamma_" + n.lower()], gamma_k=None)
        for h in range(0, x.shape[1] // d, part):
            of = slice(h * d, (h + part) * d)
            assert torch.equal(sc.rotate_forward(x[:, of], **kw1)["Q"], out[n][:, of])
            b = sc.rotate_backward(dy[:, of], None, x[:, of], **kw1)
            assert torch.equal(b["dQ"], back["d" + n][:, of])
            total[n] += b["dgamma_q"].double()
        # sums of L H products in 32 bits, in another order: each within L H 2^-24 of the sum of their sizes (a value of a normed
        # head is at most sqrt(d) before gamma)
        room = 2 * L * x.shape[1] // d * 2.0 ** -24 * float(dy.double().abs().view(-1, d).sum(0).max()) * math.sqrt(d) * 2
        assert float((total[n] - back["dgamma_" + n.lower()].double()).abs().max()) <= room


@pytest.mark.parametrize("T,H,Hk,d", [(1, 1023, 1, 64), (1, 900, 100, 128), (3, 500, 2, 64)])
def test_attend_with_many_heads(T, H, Hk, d):
    g = gen(H)
    check_attend(make_cache(g, 1, Hk, 200, d, 1, [150], BF, new=T), randn(g, T, H * d).to(BF), T, decay=0.5)


@pytest.mark.parametrize("T", [1, 20, 40])
def test_no_rows_in_use(T):
    """Nothing is attended, appended or moved; acc stays, the decay left out too."""
    g = gen(T)
    cache = make_cache(g, 3, 2, 90, 64, 2, [90, 0, 33])
    before = copy(cache)
    Q, K = randn(g, 3 * T, 128).to(BF), randn(g, 3 * T, 128).to(BF)
    got = check_attend(cache, Q, T, [0, 0, 0], decay=0.5)
    for b, n in enumerate((90, 0, 33)):
        assert torch.equal(got["acc"][b, :, :n], before["acc"][b, :, :n])
    out = {"Q": torch.full_like(Q, 3)}
    ws = sc.new_cache_workspace(3, 90, 2, 2, lists=2)
    sc.cache_append(cache, Q, K, K, L=T, rows=i32(0, 0, 0), out=out, workspace=ws)
    assert bool((out["Q"] == 3).all()) and all(same(cache[n], before[n]) for n in cache) and sc.workspace_status(ws) == sc.SC_OK


@pytest.mark.parametrize("d", [64, 128])
def test_a_cache_of_one_slot(d):
    g = gen(d)
    cache = sc.new_cache(2, 1, 2, width=d, lists=2)
    ws = sc.new_cache_workspace(2, 1, 4, 2, width=d, lists=2)
    Q, K, V = (randn(g, 2, h * d).to(BF) for h in (4, 2, 2))
    q = sc.cache_append(cache, Q, K, V, L=1, workspace=ws)["Q"]
    got = check_attend(cache, q, 1, ws=ws, in_place=True)
    assert torch.equal(got["O"].view(2, 2, 2, d), V.view(2, 2, 1, d).expand(2, 2, 2, d)) and bool((cache["acc"] == 1).all())
    check_evict(cache, budget=1)
    assert sc.workspace_status(ws) == sc.SC_OK
    sc.cache_append(cache, Q, K, V, L=1, workspace=ws)
    assert sc.workspace_status(ws) == sc.SC_ERR_CAPACITY and cache["len"].tolist() == [[1, 1], [1, 1]]
