"""Norm and rotation of heads, forward and backward, against the definition in 64 bits.

Tolerances: one rounding to the 16-bit type is half a step of it; before it, an angle is within 2^-20, so a rotated
value within 2^-20 of its pair's length, and the norm's sum of d squares in 32 bits gives (d + 32) 2^-24.  Below 2^-14
fp16 has steps of 2^-24, whatever the value: half of one is 2^-25.
"""
import itertools

import pytest
import torch

import paper_2310_07109_gb300 as sc
from cache_reference import eps_of, heads, pair_size

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
EPS = 1e-6


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def frequencies(rot, base=10000.0):
    return sc.rotary_frequencies(rot, base)[0] if rot else None


def inside(B, L, rows):
    r = torch.arange(L, device="cuda")[None, :]
    n = torch.full((B, 1), L, device="cuda") if rows is None else torch.tensor(rows, device="cuda")[:, None]
    return (r < n).reshape(-1)


CASES = [  # B, L, Hq, Hk, d, rot, interleaved, norms, rows, dtype
    (1, 1, 12, 12, 64, 64, False, "qk", None, BF),
    (1, 1, 1, 0, 16, 16, False, "", None, BF),
    (3, 37, 12, 4, 64, 64, False, "qk", [37, 0, 20], BF),
    (2, 70, 8, 2, 128, 128, True, "qk", [1, 70], HF),
    (2, 33, 4, 4, 128, 64, True, "", None, BF),
    (2, 33, 4, 4, 128, 64, False, "q", None, HF),
    (2, 19, 5, 3, 96, 32, False, "k", [19, 18], BF),
    (1, 50, 3, 1, 80, 80, False, "qk", None, HF),
    (1, 41, 2, 7, 256, 256, False, "qk", None, BF),
    (1, 41, 2, 7, 256, 16, True, "qk", [40], BF),
    (1, 23, 0, 9, 32, 32, False, "k", None, BF),
    (2, 31, 6, 6, 64, 0, False, "qk", None, BF),
    (1, 3000, 33, 17, 64, 48, False, "qk", [2999], BF),
    (4, 5000, 2, 1, 64, 64, True, "qk", None, BF),     # more tokens than warps
]


def make(case, seed=0):
    B, L, Hq, Hk, d, rot, inter, norms, rows, dt = case
    g = gen(seed + B * L + Hq + d)
    T = B * L
    # heads lie in a wider matrix, other values and, in rows not in use, NaN around them
    wide = (randn(g, T, (Hq + Hk + 1) * d) * 2).to(dt)
    used = inside(B, L, rows)
    wide[~used] = float("nan")
    Q, K = wide[:, d // 2 // 8 * 8:][:, :Hq * d], wide[:, (Hq + 1) * d:]
    pos = torch.randint(0, 100000, (B, L), device="cuda", generator=g, dtype=torch.int32)
    gam = lambda on: 1 + 0.3 * randn(g, d) if on else None  # noqa: E731
    kw = dict(width=d, B=B, L=L, rows=None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda"),
              pos=pos, freq=frequencies(rot), interleaved=inter, mscale=1.25 if rot and rot < d else 1.0,
              gamma_q=gam("q" in norms and Hq), gamma_k=gam("k" in norms and Hk), eps=EPS)
    return Q if Hq else None, K if Hk else None, kw, used


def slack_of(y, kw):
    d = kw["width"]
    y = y.reshape(y.shape[0], -1, d)
    size = pair_size(y, kw["freq"], kw["interleaved"])
    return (size * (2.0 ** -20 + (d + 32) * 2.0 ** -24)).reshape(y.shape[0], -1)


def check(got, ref, slack, used, what, u):
    got = got.double()
    bad = ~((got - ref).abs() <= u * ref.abs() * 1.01 + slack + 2.0 ** -25) & used[:, None]
    assert not bool(bad.any()), "%s: %d off, worst %.3g" % (what, int(bad.sum()), float((got - ref).abs()[bad].max()))


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    Q, K, kw, used = make(case)
    u = eps_of(case[-1])
    d = kw["width"]
    shapes = {n: (t.shape[0], t.shape[1] + 8) for n, t in (("Q", Q), ("K", K)) if t is not None}
    full = {n: torch.full(s, 7.0, dtype=case[-1], device="cuda") for n, s in shapes.items()}
    out = sc.rotate_forward(Q, K, out={n: t[:, :-8] for n, t in full.items()}, **kw)
    for n, x, gamma in (("Q", Q, kw["gamma_q"]), ("K", K, kw["gamma_k"])):
        if x is None:
            continue
        ref = heads(x, x.shape[1] // d, d, gamma, EPS, kw["pos"].reshape(-1), kw["freq"], kw["interleaved"], kw["mscale"])
        check(out[n], ref, slack_of(ref, kw), used, n, u)
        assert bool((full[n][:, -8:] == 7).all()) and bool((full[n][~used] == 7).all())


def test_forward_in_place_and_by_row():
    g = gen(5)
    x = randn(g, 2 * 9, 4 * 64).to(BF)
    kw = dict(width=64, B=2, L=9, freq=frequencies(64), gamma_q=torch.ones(64, device="cuda"))
    want = sc.rotate_forward(x, pos=torch.arange(9, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous(), **kw)["Q"]
    assert torch.equal(sc.rotate_forward(x, out={"Q": x}, **kw)["Q"], want) and torch.equal(x, want)


@pytest.mark.parametrize("inter", [False, True])
def test_far_positions(inter):
    """Every 32-bit position, negative ones too; whole turns leave nothing behind."""
    far = [0, 1, -1, 2 ** 20 + 1, 12345678, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7]
    pos = torch.tensor([far], dtype=torch.int32, device="cuda")
    x = randn(gen(3), len(far), 64).to(HF)
    freq = torch.cat([torch.tensor([1.0, 2 * torch.pi, 0.3, 1e-9], dtype=torch.float64, device="cuda"), frequencies(56)])
    kw = dict(width=64, B=1, L=len(far), pos=pos, freq=freq, interleaved=inter)
    # in the reference, whole turns are taken off in exact arithmetic
    from fractions import Fraction
    two_pi = Fraction("6.283185307179586476925286766559005768394338798750211641949889184615632812572417997256069650684234136")
    angle = [[float((p * Fraction(f)) % two_pi) for f in freq.tolist()] for p in far]
    a = torch.tensor(angle, dtype=torch.float64, device="cuda")
    first = torch.arange(0, 64, 2) if inter else torch.arange(32)
    second = first + 1 if inter else first + 32
    y = x.double()
    ref = y.clone()
    ref[:, first] = y[:, first] * a.cos() - y[:, second] * a.sin()
    ref[:, second] = y[:, second] * a.cos() + y[:, first] * a.sin()
    out = sc.rotate_forward(x, **kw)["Q"]
    size = pair_size(y[:, None], freq, inter)[:, 0]
    check(out, ref, size * 2.0 ** -19, torch.ones(len(far), dtype=torch.bool, device="cuda"), "far", eps_of(HF))


def grads(Q, K, dQ, dK, kw, used):
    """Autograd through the definition, in 64 bits."""
    d, res = kw["width"], {}
    for n, x, dy, gamma in (("Q", Q, dQ, kw["gamma_q"]), ("K", K, dK, kw["gamma_k"])):
        if dy is None:
            continue
        x = torch.where(used[:, None], x.double(), 0.5).requires_grad_(True)
        gamma = None if gamma is None else gamma.double().requires_grad_(True)
        y = heads(x, x.shape[1] // d, d, gamma, EPS, kw["pos"].reshape(-1), kw["freq"], kw["interleaved"], kw["mscale"])
        got = torch.autograd.grad(y, [x] + ([] if gamma is None else [gamma]), torch.where(used[:, None], dy.double(), 0.0))
        res["d" + n] = got[0]
        if gamma is not None:
            res["dgamma_" + n.lower()] = got[1]
    return res


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    B, L, Hq, Hk, d, rot, inter, norms, rows, dt = case
    Q, K, kw, used = make(case)
    g = gen(77)
    dy = {n: randn(g, B * L, h * d).to(dt) for n, h in (("dQ", Hq), ("dK", Hk)) if h}
    for t in dy.values():
        t[~used] = float("nan")
    out = {n: torch.full_like(t, 7.0) for n, t in dy.items()}
    for n, gamma in (("dgamma_q", kw["gamma_q"]), ("dgamma_k", kw["gamma_k"])):
        if gamma is not None:
            out[n] = torch.empty(d, device="cuda")
    got = sc.rotate_backward(dy.get("dQ"), dy.get("dK"), Q, K, out=out, **kw)
    ref = grads(Q, K, dy.get("dQ"), dy.get("dK"), kw, used)
    assert set(got) == set(ref)
    u = eps_of(dt)
    for n, r in ref.items():
        if n.startswith("dgamma"):
            # sums of T H products in 32 bits: one after the other within a lane, whose own are at most
            # ceil(T / warps) ceil(H / heads at once); then lanes, warps, CTAs
            x = Q if n.endswith("q") else K
            size = torch.nan_to_num(torch.where(used[:, None], dy["dQ" if n.endswith("q") else "dK"].double(), 0.0)).abs()
            size = (size.reshape(-1, d).sum(0) * kw["mscale"] * 2).max()
            xh = torch.where(used[:, None], x.double(), 0.0).reshape(-1, d)
            hat = (xh / torch.sqrt((xh * xh).mean(-1, keepdim=True) + EPS)).abs().max()
            terms = B * L * max(Hq, Hk) / 64 + 64
            assert float((got[n].double() - r).abs().max()) <= float(size * hat) * (2.0 ** -20 + (terms + d) * 2.0 ** -24), n
            continue
        # a gradient is inv (dy gamma - h mean(dy gamma h)): each term's errors against the sum of their sizes
        x = (Q if n == "dQ" else K)
        h = torch.where(used[:, None], x.double(), 0.5).reshape(B * L, -1, d)
        dyd = torch.where(used[:, None], dy[n].double(), 0.0).reshape(B * L, -1, d)
        gamma = kw["gamma_q"] if n == "dQ" else kw["gamma_k"]
        size = pair_size(dyd, kw["freq"], inter) * kw["mscale"]
        if gamma is not None:
            inv = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)
            size = size * gamma.double().abs()
            hat = (h * inv).abs()
            size = inv * (size + hat * (size * hat).mean(-1, keepdim=True))
        slack = (size * (2.0 ** -20 + (2 * d + 64) * 2.0 ** -24)).reshape(B * L, -1)
        check(got[n], r, slack, used, n, u)
        assert bool((got[n][~used] == 7).all())


def test_backward_against_differences():
    """The slope of a sum of the outputs along a random direction, by central differences of the 64-bit definition."""
    case = (2, 21, 4, 2, 64, 32, True, "qk", [21, 13], HF)
    Q, K, kw, used = make(case)
    g = gen(9)
    d = 64
    Q, K = (torch.where(used[:, None], t, 0).contiguous() for t in (Q, K))
    dQ, dK = randn(g, 42, 4 * d).to(HF), randn(g, 42, 2 * d).to(HF)
    got = sc.rotate_backward(dQ, dK, Q, K, **kw)
    for n, x, dy, gamma in (("q", Q, dQ, kw["gamma_q"]), ("k", K, dK, kw["gamma_k"])):
        weight = torch.where(used[:, None], dy.double(), 0.0)
        f = lambda x, gm: (weight * heads(x, x.shape[1] // d, d, gm, EPS, kw["pos"].reshape(-1), kw["freq"],  # noqa: E731
                                          True, kw["mscale"])).sum()
        step = 1e-5
        v = torch.where(used[:, None], randn(g, *x.shape).double(), 0.0)
        slope = (f(x.double() + step * v, gamma) - f(x.double() - step * v, gamma)) / (2 * step)
        dx = torch.where(used[:, None], got["d" + n.upper()].double(), 0.0)
        room = float((dx * v).abs().sum()) * (eps_of(HF) * 1.1) + 1e-6 * float(weight.abs().sum())
        assert abs(float(slope - (dx * v).sum())) <= room
        w = randn(g, d).double()
        slope = (f(x.double(), gamma.double() + step * w) - f(x.double(), gamma.double() - step * w)) / (2 * step)
        assert abs(float(slope - (got["dgamma_" + n].double() * w).sum())) <= 1e-5 * float(weight.abs().sum())


def test_backward_undoes_the_rotation():
    """Without a norm the gradient is the rotation by -p (and mscale)."""
    g = gen(4)
    y = randn(g, 64, 8 * 64).to(BF)
    pos = torch.randint(0, 1 << 20, (1, 64), device="cuda", generator=g, dtype=torch.int32)
    kw = dict(width=64, B=1, L=64, freq=frequencies(64))
    back = sc.rotate_backward(y, pos=pos, **kw)["dQ"]
    assert torch.equal(back, sc.rotate_forward(y, pos=(-pos).contiguous(), **kw)["Q"])


def test_tokens_far_apart_in_memory():
    """More than 2^31 elements between the first token and the last."""
    T, ld = 2500, 1 << 20
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    x = torch.empty(T * ld, dtype=BF, device="cuda").as_strided((T, 128), (ld, 1))
    x.copy_(randn(gen(8), T, 128))
    kw = dict(width=64, B=1, L=T, freq=frequencies(64), gamma_q=torch.ones(64, device="cuda"))
    want, dy = sc.rotate_forward(x.contiguous(), **kw)["Q"], randn(gen(9), T, 128).to(BF)
    back = sc.rotate_backward(dy, None, x.contiguous(), **kw)
    got = sc.rotate_backward(dy, None, x, **kw)
    assert all(torch.equal(back[n], got[n]) for n in back)
    assert torch.equal(sc.rotate_forward(x, out={"Q": x}, **kw)["Q"], want)


def test_two_calls_give_the_same_bits():
    case = (4, 700, 12, 4, 64, 64, False, "qk", [700, 3, 0, 512], BF)
    Q, K, kw, used = make(case)
    dQ, dK = randn(gen(1), 2800, 12 * 64).to(BF), randn(gen(2), 2800, 4 * 64).to(BF)
    a, b = (sc.rotate_backward(dQ, dK, Q, K, **kw) for _ in range(2))
    assert torch.equal(a["dgamma_q"], b["dgamma_q"]) and torch.equal(a["dgamma_k"], b["dgamma_k"])


def test_in_a_graph_with_other_rows_and_positions():
    case = (2, 40, 4, 4, 64, 64, False, "qk", [40, 40], BF)
    Q, K, kw, _ = make(case)
    Q, K = Q.contiguous(), K.contiguous()
    ws = sc.new_rotate_workspace(64)
    dQ, dK = torch.ones_like(Q), torch.ones_like(K)
    out = sc.rotate_forward(Q, K, **kw)
    back = sc.rotate_backward(dQ, dK, Q, K, workspace=ws, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sc.rotate_forward(Q, K, out=out, **kw)
        sc.rotate_backward(dQ, dK, Q, K, out=back, workspace=ws, **kw)
    g = gen(12)
    for rows in ([40, 17], [0, 1]):
        for t in (Q, K, dQ, dK):
            t.copy_(randn(g, *t.shape))
        kw["rows"].copy_(torch.tensor(rows))
        kw["pos"].copy_(torch.randint(0, 1000, (2, 40), device="cuda", generator=g))
        graph.replay()
        fwd, bwd = sc.rotate_forward(Q, K, **kw), sc.rotate_backward(dQ, dK, Q, K, **kw)
        used = inside(2, 40, rows)
        for n in ("Q", "K"):
            assert torch.equal(out[n][used], fwd[n][used]) and torch.equal(back["d" + n][used], bwd["d" + n][used])
            assert torch.equal(back["dgamma_" + n.lower()], bwd["dgamma_" + n.lower()])


def test_on_another_stream():
    case = (2, 300, 12, 4, 64, 64, False, "qk", None, BF)
    Q, K, kw, _ = make(case)
    Q, K = Q.contiguous(), K.contiguous()
    want = sc.rotate_forward(Q, K, **kw)
    back = sc.rotate_backward(Q, K, Q, K, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, got_back = sc.rotate_forward(Q, K, stream=side, **kw), sc.rotate_backward(Q, K, Q, K, stream=side, **kw)
    side.synchronize()
    for a, b in itertools.chain(((got[n], want[n]) for n in want), ((got_back[n], back[n]) for n in back)):
        assert torch.equal(a, b)


def test_backward_without_a_norm_makes_nothing_of_q_and_k():
    """Q and K are not used without a norm: no address and distance given for them matters, odd ones included."""
    import ctypes

    from paper_2310_07109_gb300 import binding, cache

    B, L, Hq, Hk, d = 2, 21, 5, 2, 96
    g = gen(5)
    dQ, dK = randn(g, B * L, Hq * d).to(BF), randn(g, B * L, Hk * d).to(BF)
    freq, gamma = frequencies(32), 1 + 0.3 * randn(g, d)
    X = randn(g, B * L, Hq * d).to(BF)
    ws = sc.new_rotate_workspace(d)
    for norm in (False, True):   # of the queries; the keys have none
        want = sc.rotate_backward(dQ, dK, X if norm else None, width=d, B=B, L=L, freq=freq, gamma_q=gamma if norm else None, workspace=ws)
        got = {n: torch.full_like(t, float("nan")) for n, t in want.items()}
        a = cache.RotateBackwardArgs(
            B=B, L=L, Hq=Hq, Hk=Hk, d=d, dtype=0, dQ_out=dQ.data_ptr(), ldq_out=Hq * d, dK_out=dK.data_ptr(), ldk_out=Hk * d,
            Q=X.data_ptr() if norm else 3, ldq=Hq * d if norm else 5, K=3, ldk=7, gamma_q=gamma.data_ptr() if norm else None,
            eps=EPS, rot=32, freq=freq.data_ptr(), mscale=1.0, dQ=got["dQ"].data_ptr(), ldq_grad=Hq * d, dK=got["dK"].data_ptr(),
            ldk_grad=Hk * d, dgamma_q=got["dgamma_q"].data_ptr() if norm else None)
        rc = binding.load().sc_rotate_backward(ctypes.byref(a), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        for n in want:
            assert torch.equal(got[n], want[n]), n
