"""The expert feed-forward operators against plain 64-bit evaluations: routing, products
grouped by expert and the gated sum with residual and layer norm, forward and backward.

Tolerances come from the arithmetic.  A value rounded once to bf16 (8 significant bits) is within
2^-8 of itself.  A sum of C products in fp32, in any order and
with truncated additions, is within (C + 16) 2^-23 of the sum of their magnitudes.  The
GELU used may be 2e-7 off per unit of its argument (its erf is a published
approximation with 1.5e-7).
"""
import math

import pytest
import torch

import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu

U_BF16 = 2.0 ** -8
U_F32 = 2.0 ** -23


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def bf16(t):
    return t.to(torch.bfloat16)


def check(got, ref, slack, rounding, what):
    """|got - ref| <= rounding |ref| + slack, elementwise; no NaN where ref has none."""
    got = got.double()
    assert got.shape == ref.shape
    bad = ~((got - ref).abs() <= rounding * ref.abs() * 1.01 + slack)
    assert not bool(bad.any()), "%s: %d of %d off, worst %.3g against %.3g" % (
        what, int(bad.sum()), bad.numel(), float((got - ref).abs()[bad].max()),
        float(ref.abs()[bad].max()))


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------
def route_ref(logits, lens, B, L, k, renorm):
    """One token at a time on the host, in 64 bits."""
    x = logits.double().cpu()
    T, E = x.shape
    expert = torch.full((T, k), -1, dtype=torch.int32)
    gate = torch.zeros(T, k, dtype=torch.float64)
    by = [[] for _ in range(E)]
    for t in range(T):
        if t % L >= lens[t // L]:
            continue
        row = [-math.inf if math.isnan(v) else v for v in x[t].tolist()]
        order = sorted((e for e in range(E) if row[e] > -math.inf), key=lambda e: (-row[e], e))[:k]
        if not order:
            continue
        m = row[order[0]]
        ex = [1.0 if v == m else math.exp(v - m) for v in row]
        total = sum(ex[e] for e in order) if renorm else sum(ex)
        for j, e in enumerate(order):
            expert[t, j] = e
            gate[t, j] = ex[e] / total
            by[e].append((t, j))
    offsets, slot, token = [0], torch.full((T, k), -1, dtype=torch.int32), []
    for e in range(E):
        for t, j in by[e]:
            slot[t, j] = len(token)
            token.append(t)
        offsets.append(len(token))
    token += [-1] * (T * k - len(token))
    return expert, gate, torch.tensor(offsets, dtype=torch.int32), slot, torch.tensor(token, dtype=torch.int32)


def route_logits(g, T, E, kind):
    x = randn(g, T, E)
    if kind == "ties":
        x = (x * 2).round() / 2
    elif kind == "masked":
        x[torch.rand((T, E), device="cuda", generator=g) < 0.5] = -math.inf
        x[::3] = -math.inf                                     # whole rows masked
    elif kind == "extremes":
        pick = torch.randint(0, 6, (T, E), device="cuda", generator=g)
        low, high = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
        for i, v in enumerate((math.nan, math.inf, -math.inf, low, high)):
            x[pick == i] = v
        x[::5] = low                                           # the lowest value everywhere: not masked
        x[1::5] = math.nan
    elif kind == "signed zeros":
        x = torch.where(x > 0, 0.0, -0.0)
    return x


@pytest.mark.parametrize("B,L,E,k,rows,kind", [
    (1, 1, 8, 2, None, "plain"),
    (1, 1, 1, 1, None, "plain"),
    (3, 50, 16, 2, [0, 50, 17], "ties"),
    (2, 64, 33, 8, None, "masked"),
    (1, 127, 64, 4, None, "extremes"),
    (1, 129, 256, 8, [128], "masked"),
    (2, 200, 7, 7, [200, 3], "signed zeros"),
    (4, 130, 100, 3, [0, 0, 0, 0], "plain"),
    (1, 3000, 12, 2, [2999], "ties"),
    (2, 20000, 5, 1, [20000, 19000], "masked"),     # several chunks of tokens a CTA
])
@pytest.mark.parametrize("renorm", [True, False])
def test_route(B, L, E, k, rows, kind, renorm):
    g = gen(B * 1000 + L + E + k)
    T = B * L
    wide = torch.full((T, E + 5), math.inf, device="cuda")
    wide[:, :E] = route_logits(g, T, E, kind)
    logits = wide[:, :E]                                       # rows further apart than E
    lens = rows if rows is not None else [L] * B
    rows_t = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    ref = route_ref(logits, lens, B, L, k, renorm)
    got = sc.expert_route_forward(logits, k=k, B=B, L=L, rows=rows_t, renormalize=renorm)
    for name, r in zip(("expert", "offsets", "slot", "token"), (ref[0], ref[2], ref[3], ref[4])):
        assert torch.equal(got[name].cpu(), r), name
    # expf, a sum of at most E terms and a division: (E + 8) roundings
    check(got["gate"].cpu(), ref[1], 1e-38, (E + 8) * U_F32, "gate")
    again = sc.expert_route_forward(logits, k=k, B=B, L=L, rows=rows_t, renormalize=renorm)
    for name in got:
        assert torch.equal(got[name], again[name]), name


@pytest.mark.parametrize("B,L,E,k,rows,kind", [
    (1, 1, 8, 2, None, "plain"), (2, 65, 33, 8, [65, 9], "masked"), (1, 300, 64, 4, None, "ties"),
    (1, 100, 200, 3, None, "extremes"), (3, 7, 2, 1, [0, 7, 2], "plain")])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward(B, L, E, k, rows, kind, renorm):
    g = gen(7 + B * L + E)
    T = B * L
    logits = route_logits(g, T, E, kind)
    rows_t = None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda")
    r = sc.expert_route_forward(logits, k=k, B=B, L=L, rows=rows_t, renormalize=renorm)
    dgate = randn(g, T, k)
    dgate[r["expert"] < 0] = math.nan                          # no choice: not read
    got = sc.expert_route_backward(logits, r["expert"], r["gate"], dgate, B=B, L=L, rows=rows_t,
                                   renormalize=renorm)
    # softmax Jacobian in 64 bits
    x = torch.where(logits.isnan(), -math.inf, logits).double()
    chosen = torch.zeros(T, E, dtype=torch.bool, device="cuda")
    dg = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    for j in range(k):
        ok = r["expert"][:, j] >= 0
        e = r["expert"][ok, j].long()
        chosen[ok, e] = True
        dg[ok, e] = dgate[ok, j].double()
    some = chosen.any(dim=1)
    m = x.amax(dim=1, keepdim=True)
    ex = torch.where(x == m, 1.0, torch.exp(x - m))
    ex = torch.where(chosen if renorm else x > -math.inf, ex, 0.0)
    p = torch.where(some[:, None], ex / ex.sum(dim=1, keepdim=True), 0.0)
    ref = torch.where(some[:, None], p * (dg - (p * dg).sum(dim=1, keepdim=True)), 0.0)
    big = (p * dg.abs()).sum(dim=1, keepdim=True) + dg.abs()
    check(got, ref, (E + 16) * U_F32 * p * big + 1e-38, 0.0, "dlogits")
    assert bool((got[~some] == 0).all())


@pytest.mark.parametrize("E", [2, 8, 9, 16, 17, 24, 32, 33, 64, 65, 128, 129, 255, 256])
@pytest.mark.parametrize("kind", ["ties", "masked", "extremes"])
def test_route_of_every_number_of_experts(E, kind):
    test_route(2, 133, E, min(E, 8), [133, 70], kind, E % 2 == 0)


def test_route_backward_is_the_difference_quotient():
    """Where the choice does not change, dlogits is the gates' slope (differences in 64 bits)."""
    T, E, k, h = 6, 9, 3, 1e-4
    x = randn(gen(3), T, E)
    w = randn(gen(4), T, k)
    for renorm in (True, False):
        r = sc.expert_route_forward(x, k=k, B=1, L=T, renormalize=renorm)
        d = sc.expert_route_backward(x, r["expert"], r["gate"], w, B=1, L=T, renormalize=renorm)
        pick = r["expert"].long()

        def f(y):
            z = torch.gather(y, 1, pick) if renorm else y
            p = torch.softmax(z, dim=1)
            return ((p if renorm else torch.gather(p, 1, pick)) * w.double()).sum(dim=1)

        for e in range(E):
            step = torch.zeros(T, E, dtype=torch.float64, device="cuda")
            step[:, e] = h
            slope = (f(x.double() + step) - f(x.double() - step)) / (2 * h)
            # the quotient is off by h^2 / 6 of the third derivative (at most 3 |w|)
            check(d[:, e].cpu(), slope.cpu(), 1e-6, 0.0, "slope")


# ---------------------------------------------------------------------------
# products grouped by expert
# ---------------------------------------------------------------------------
def offsets_of(counts, first=0):
    return torch.tensor([first] + counts, device="cuda").cumsum(0).int()


def gelu64(x):
    return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))


def gelu_slope64(x):
    return 0.5 * (1 + torch.erf(x / math.sqrt(2))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


# (slots of each expert, N, K)
SHAPES = [
    ([1], 8, 8),
    ([0, 1, 0], 16, 24),
    ([2, 0, 1, 1], 768, 512),                       # a few slots: one token's experts
    ([5, 3, 0, 7, 1], 264, 136),
    ([16, 16], 72, 1032),
    ([17, 31, 32, 33], 136, 200),
    ([0, 0, 0], 64, 64),                            # nothing routed at all
    ([127, 128, 129, 0, 1, 63, 64, 65], 520, 264),
    ([255, 256, 257, 300], 256, 64),
    ([700, 0, 3, 1100], 1000, 328),
    ([40] * 64, 512, 256),
    ([3, 2, 1, 0] * 64, 128, 192),                  # the most experts
    ([513], 2048, 768),
]


def product_inputs(seed, counts, rows, width, *, gather, pad, first=0, spare=5):
    """Rows for the slots; what no slot may read is NaN."""
    g = gen(seed)
    M = first + sum(counts) + spare
    n = rows if gather else M
    buf = torch.full((n, width + pad), math.nan, device="cuda", dtype=torch.bfloat16)
    x = buf[:, :width]
    x.copy_(bf16(randn(g, n, width)))
    token = None
    if gather:
        token = torch.full((M,), -1, dtype=torch.int32, device="cuda")
        token[first: M - spare] = torch.randint(0, n, (M - spare - first,), device="cuda", generator=g).int()
    else:
        x[:first] = math.nan
        x[M - spare:] = math.nan
    return x, token, M


@pytest.mark.parametrize("counts,N,K", SHAPES)
@pytest.mark.parametrize("gather,pad,gelu,pre,f32,bias,first", [
    (True, 0, True, True, False, True, 0),
    (False, 8, False, False, True, False, 3),
    (True, 24, True, False, True, True, 2),
    (False, 0, False, True, False, True, 0),
    (False, 16, True, True, True, True, 1),
])
def test_expert_linear_forward(counts, N, K, gather, pad, gelu, pre, f32, bias, first):
    E = len(counts)
    X, token, M = product_inputs(11 + N + K, counts, 97, K, gather=gather, pad=pad, first=first)
    g = gen(N * K)
    W = bf16(randn(g, E, N, K) / math.sqrt(K))
    b = randn(g, E, N) if bias else None
    off = offsets_of(counts, first)
    out = torch.full((M, N), -7.0, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    prev = torch.full((M, N), -9.0, device="cuda", dtype=torch.bfloat16) if pre else None
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    sc.expert_linear_forward(X, W, off, token=token, bias=b, gelu=gelu, pre=prev, out=out, workspace=ws)
    assert sc.workspace_status(ws) == 0
    lo = first
    for e, c in enumerate(counts):
        hi = lo + c
        rows = X[lo:hi] if token is None else X[token[lo:hi].long()]
        rows, w = rows.double(), W[e].double()
        y = rows @ w.T + (b[e].double() if bias else 0.0)
        slack = (K + 16) * U_F32 * (rows.abs() @ w.abs().T + (b[e].abs().double() if bias else 0.0))
        ref = gelu64(y) if gelu else y
        # GELU's slope is at most 1.13
        check(out[lo:hi], ref, 1.13 * slack + (4e-7 * (1 + y.abs()) if gelu else 0.0),
              U_F32 if f32 else U_BF16, "expert %d" % e)
        if pre:
            check(prev[lo:hi], y, slack, U_BF16, "pre, expert %d" % e)
        lo = hi
    used = torch.zeros(M, dtype=torch.bool, device="cuda")
    used[first:lo] = True
    assert bool((out[~used] == -7.0).all()), "slots past the ones in use were written"
    assert prev is None or bool((prev[~used] == -9.0).all())
    again = torch.full_like(out, -7.0)
    sc.expert_linear_forward(X, W, off, token=token, bias=b, gelu=gelu, out=again, workspace=ws)
    assert torch.equal(again, out)


@pytest.mark.parametrize("counts,N,K", SHAPES)
@pytest.mark.parametrize("pad,pre,f32,first", [(0, True, False, 0), (16, False, True, 4), (8, True, True, 1)])
def test_expert_linear_backward_input(counts, N, K, pad, pre, f32, first):
    E = len(counts)
    dY, _, M = product_inputs(5 + N + K, counts, 0, N, gather=False, pad=pad, first=first)
    g = gen(N + 3 * K)
    W = bf16(randn(g, E, N, K) / math.sqrt(N))
    z = bf16(2 * randn(g, M, K)) if pre else None
    off = offsets_of(counts, first)
    out = torch.full((M, K), -7.0, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    sc.expert_linear_backward_input(dY, W, off, pre=z, out=out, workspace=ws)
    assert sc.workspace_status(ws) == 0
    lo = first
    for e, c in enumerate(counts):
        hi = lo + c
        dy, w = dY[lo:hi].double(), W[e].double()
        ref, mag = dy @ w, dy.abs() @ w.abs()
        slack = (N + 16) * U_F32 * mag
        if pre:
            s = gelu_slope64(z[lo:hi].double())
            slack = 1.13 * slack + 1e-6 * ref.abs()
            ref = ref * s
        check(out[lo:hi], ref, slack, U_F32 if f32 else U_BF16, "expert %d" % e)
        lo = hi
    used = torch.zeros(M, dtype=torch.bool, device="cuda")
    used[first:lo] = True
    assert bool((out[~used] == -7.0).all())


@pytest.mark.parametrize("counts,N,K", SHAPES)
@pytest.mark.parametrize("gather,pad,f32,bias,first", [(True, 0, True, True, 0), (False, 8, False, True, 3),
                                                       (True, 16, False, False, 2)])
def test_expert_linear_backward_weight(counts, N, K, gather, pad, f32, bias, first):
    E = len(counts)
    X, token, M = product_inputs(2 + N + K, counts, 97, K, gather=gather, pad=pad, first=first)
    dY, _, _ = product_inputs(3 + N + K, counts, 0, N, gather=False, pad=pad, first=first)
    off = offsets_of(counts, first)
    out = {"dW": torch.full((E, N, K), math.nan, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)}
    if bias:
        out["dbias"] = torch.full((E, N), math.nan, device="cuda")
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    sc.expert_linear_backward_weight(dY, X, off, token=token, out=out, workspace=ws)
    assert sc.workspace_status(ws) == 0
    lo = first
    for e, c in enumerate(counts):
        hi = lo + c
        rows = (X[lo:hi] if token is None else X[token[lo:hi].long()]).double()
        dy = dY[lo:hi].double()
        slack = (c + 16) * U_F32 * (dy.abs().T @ rows.abs())
        check(out["dW"][e], dy.T @ rows, slack, U_F32 if f32 else U_BF16, "dW, expert %d" % e)
        if bias:
            check(out["dbias"][e], dy.sum(dim=0), (c + 16) * U_F32 * dy.abs().sum(dim=0), 0.0,
                  "dbias, expert %d" % e)
        lo = hi
    again = sc.expert_linear_backward_weight(dY, X, off, token=token, out_f32=f32, bias=bias, workspace=ws)
    for name in out:
        assert torch.equal(again[name], out[name]), name


@pytest.mark.parametrize("E", [19, 20, 38, 58, 59, 60, 77])
@pytest.mark.parametrize("f32", [True, False])
def test_expert_linear_backward_weight_writes_every_tile(E, f32):
    """Uneven experts of four tiles each, around one and three tiles for each pair of SMs."""
    N, K = 1000, 200
    counts = [(0, 1, 700, 64, 65, 3, 1900, 0, 130, 15, 400)[(7 * e) % 11] for e in range(E)]
    X, token, M = product_inputs(5 + E, counts, 301, K, gather=f32, pad=0)
    dY, _, _ = product_inputs(6 + E, counts, 0, N, gather=False, pad=0)
    off = offsets_of(counts)
    out = {"dW": torch.full((E, N, K), math.nan, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16),
           "dbias": torch.full((E, N), math.nan, device="cuda")}
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    sc.expert_linear_backward_weight(dY, X, off, token=token, out=out, workspace=ws)
    assert sc.workspace_status(ws) == 0
    lo = 0
    for e, c in enumerate(counts):
        hi = lo + c
        rows = (X[lo:hi] if token is None else X[token[lo:hi].long()]).double()
        dy = dY[lo:hi].double()
        slack = (c + 16) * U_F32 * (dy.abs().T @ rows.abs())
        check(out["dW"][e], dy.T @ rows, slack, U_F32 if f32 else U_BF16, "dW, expert %d" % e)
        check(out["dbias"][e], dy.sum(dim=0), (c + 16) * U_F32 * dy.abs().sum(dim=0), 0.0, "dbias, expert %d" % e)
        lo = hi


def test_expert_linear_keeps_rows_apart():
    """A row of infinities or NaN reaches its own outputs alone."""
    counts, N, K = [60, 70, 130], 200, 136
    X, _, M = product_inputs(1, counts, 0, K, gather=False, pad=0, spare=0)
    W = bf16(randn(gen(2), 3, N, K))
    off = offsets_of(counts)
    clean = sc.expert_linear_forward(X, W, off)
    bad = X.clone()
    bad[59], bad[60], bad[200] = math.nan, math.inf, math.nan
    got = sc.expert_linear_forward(bad, W, off)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[[59, 60, 200]] = False
    assert torch.equal(got[keep], clean[keep])
    assert not bool(torch.isfinite(got[~keep].float()).any())
    # and in the weight gradient a bad row spoils its own expert alone
    dY = bf16(randn(gen(3), M, N))
    clean = sc.expert_linear_backward_weight(dY, X, off)
    bad = X.clone()
    bad[60] = math.nan
    got = sc.expert_linear_backward_weight(dY, bad, off)
    assert torch.equal(got["dW"][[0, 2]], clean["dW"][[0, 2]])
    assert bool(got["dW"][1].isnan().all())


def test_expert_linear_offsets_out_of_range():
    """Offsets and tokens outside their ranges are held inside them: nothing else is touched."""
    M, N, K, rows = 40, 64, 72, 11
    g = gen(1)
    X, W = bf16(randn(g, rows, K)), bf16(randn(g, 3, N, K))
    off = torch.tensor([-5, 25, 20, 90], dtype=torch.int32, device="cuda")     # not even in order
    token = torch.tensor([-1, rows, 1 << 30] + [3] * (M - 3), dtype=torch.int32, device="cuda")
    guard = torch.full((M + 2, N), 5.0, device="cuda", dtype=torch.bfloat16)
    ws = sc.new_expert_workspace(1, 1, 1, 1, 8)
    sc.expert_linear_forward(X, W, off, token=token, out=guard[1:-1], workspace=ws)
    sc.expert_linear_backward_weight(bf16(randn(g, M, N)), X, off, token=token, workspace=ws)
    assert sc.workspace_status(ws) == 0
    assert bool((guard[0] == 5).all()) and bool((guard[-1] == 5).all())
    want = X[3].double() @ W[0].double().T
    check(guard[11], want, (K + 16) * U_F32 * (X[3].double().abs() @ W[0].double().abs().T), U_BF16, "slot 10")


@pytest.mark.parametrize("M", [1, 7, 16, 17])
@pytest.mark.parametrize("gelu,pre,f32", [(True, True, False), (False, False, True)])
def test_expert_linear_few_slots(M, gelu, pre, f32):
    """Around the number of slots below which another kernel runs, some of them not in use."""
    E, N, K = 40, 152, 264
    g = gen(M)
    X, W, b = bf16(randn(g, 5, K)), bf16(randn(g, E, N, K) / 16), randn(g, E, N)
    used = max(1, M - 2)
    pick = torch.randint(0, E, (used,), device="cuda", generator=g).sort().values
    off = torch.searchsorted(pick, torch.arange(E + 1, device="cuda")).int()
    token = torch.randint(0, 5, (M,), device="cuda", generator=g).int()
    out = torch.full((M, N), -7.0, device="cuda", dtype=torch.float32 if f32 else torch.bfloat16)
    prev = torch.full((M, N), -9.0, device="cuda", dtype=torch.bfloat16) if pre else None
    sc.expert_linear_forward(X, W, off, token=token, bias=b, gelu=gelu, pre=prev, out=out)
    x = X[token[:used].long()].double()
    y = torch.einsum("sk,snk->sn", x, W[pick].double()) + b[pick].double()
    slack = (K + 16) * U_F32 * (torch.einsum("sk,snk->sn", x.abs(), W[pick].double().abs()) + b[pick].abs().double())
    check(out[:used], gelu64(y) if gelu else y, 1.13 * slack + (4e-7 * (1 + y.abs()) if gelu else 0.0),
          U_F32 if f32 else U_BF16, "out")
    assert bool((out[used:] == -7.0).all())
    if pre:
        check(prev[:used], y, slack, U_BF16, "pre")
        assert bool((prev[used:] == -9.0).all())


def test_gelu_of_infinities_and_nan():
    """Values that overflow, and NaN, next to ordinary ones: each stays its own."""
    N, K, M = 64, 64, 40
    W = torch.zeros(1, N, K, device="cuda", dtype=torch.bfloat16)
    W[0, :, 0] = 1
    vals = torch.tensor([math.inf, 1.0, -math.inf, -1.0, math.nan, 2.0, 3e38, -2.0, -3e38, 0.5], device="cuda")
    X = torch.zeros(M, K, device="cuda", dtype=torch.bfloat16)
    X[:, 0] = bf16(vals.repeat(4))
    off = offsets_of([M])
    want = torch.nn.functional.gelu(X[:, :1].double()).expand(M, N)
    want = torch.where(X[:, :1].isinf() & (X[:, :1] < 0), 0.0, want)       # the limit, where the product is NaN
    for rows in (M, 10):                                                   # both kernels
        got = sc.expert_linear_forward(X[:rows], W, offsets_of([rows]), gelu=True).double()
        ref = want[:rows]
        assert bool((got.isnan() == ref.isnan()).all())
        fin = ~ref.isnan()
        same = (got == ref) | ((got - ref).abs() <= U_BF16 * ref.abs() + 1e-6)
        assert bool(same[fin].all())


@pytest.mark.parametrize("rows", [250, 16])
def test_gelu_and_its_slope_beside_outliers(rows):
    """Ordinary values whose neighbours are far out (the arithmetic runs on pairs)."""
    N, K = 64, 64
    x = torch.linspace(-7, 7, rows, device="cuda")
    x[1::2] = torch.tensor([100.0, -9.0, 3e4, -1e6, 8.0], device="cuda").repeat(rows)[: rows // 2]
    for shift in (0, 1):
        X = torch.zeros(rows, K, device="cuda", dtype=torch.bfloat16)
        X[:, 0] = bf16(x.roll(shift))
        W = torch.zeros(1, N, K, device="cuda", dtype=torch.bfloat16)
        W[0, :, 0] = 1
        v = X[:, :1].double().expand(rows, N)
        got = sc.expert_linear_forward(X, W, offsets_of([rows]), gelu=True, out_f32=True)
        check(got, gelu64(v), 4e-7 * (1 + v.abs().clamp(max=10)), U_F32, "gelu")
        pre = X[:, :1].expand(rows, K).contiguous()
        dY = torch.zeros(rows, N, device="cuda", dtype=torch.bfloat16)
        dY[:, 0] = 1
        one = torch.zeros(1, N, K, device="cuda", dtype=torch.bfloat16)
        one[0, 0] = 1
        got = sc.expert_linear_backward_input(dY, one, offsets_of([rows]), pre=pre, out_f32=True)
        check(got, gelu_slope64(pre.double()), 2e-6, U_F32, "slope")


def test_expert_linear_on_another_stream():
    """Without a workspace given, and on a stream that is not the current one."""
    counts, N, K = [300, 20, 411], 256, 320
    X, _, _ = product_inputs(1, counts, 0, K, gather=False, pad=0, spare=0)
    W = bf16(randn(gen(2), 3, N, K))
    off = offsets_of(counts)
    ref = sc.expert_linear_forward(X, W, off)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(ref)
    out.record_stream(side)
    sc.expert_linear_forward(X, W, off, out=out, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, ref)


def test_outputs_made_for_another_stream():
    """Memory that the current stream still writes when a call on another stream is given it."""
    rows, E, N, K = 4096, 2, 1024, 64
    X, W = bf16(randn(gen(3), rows, K)), bf16(randn(gen(4), E, N, K))
    off = offsets_of([1000, 3096])
    logits = randn(gen(5), rows, 16)
    ref = sc.expert_linear_forward(X, W, off)
    ref_route = sc.expert_route_forward(logits, k=2, B=1, L=rows)
    ws = sc.new_expert_workspace(1, rows, 16, 2, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = {}
    torch.cuda.synchronize()
    for name, call, nbytes in (
            ("linear", lambda: {"out": sc.expert_linear_forward(X, W, off, workspace=ws, stream=side)}, rows * N * 2),
            ("route", lambda: sc.expert_route_forward(logits, k=2, B=1, L=rows, workspace=ws, stream=side), rows * 8)):
        busy = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in range(4)]
        big = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        for i in range(40):
            big.fill_(i)
        for t in busy:
            t.fill_(7)
        del busy, t
        got[name] = call()
    torch.cuda.synchronize()
    assert torch.equal(got["linear"]["out"], ref)
    for name in ref_route:
        assert torch.equal(got["route"][name], ref_route[name]), name


def test_expert_products_in_a_graph():
    """Captured, and replayed with other rows, another routing and other lengths."""
    T, E, k, D, F = 200, 8, 2, 256, 512
    g = gen(9)
    X, W, b = bf16(randn(g, T, D)), bf16(randn(g, E, F, D) / 16), randn(g, E, F)
    logits = randn(g, T, E)
    rows = torch.tensor([T], dtype=torch.int32, device="cuda")
    ws = sc.new_expert_workspace(1, T, E, k, F)

    def block():
        r = sc.expert_route_forward(logits, k=k, B=1, L=T, rows=rows, workspace=ws)
        return r, sc.expert_linear_forward(X, W, r["offsets"], token=r["token"], bias=b, gelu=True, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            r, out = block()
    torch.cuda.synchronize()
    for n in (T, 57, 1, 0):
        X.copy_(bf16(randn(g, T, D)))
        logits.copy_(randn(g, T, E))
        rows.fill_(n)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        r2, want = block()
        used = int(r2["offsets"][-1])
        assert used == k * n
        assert torch.equal(r["slot"], r2["slot"]) and torch.equal(r["token"], r2["token"])
        assert torch.equal(out[:used], want[:used])
        assert bool((out[used:] == 0).all())


# ---------------------------------------------------------------------------
# gated sum, residual, layer norm
# ---------------------------------------------------------------------------
def combine_inputs(seed, B, L, D, k, rows):
    g = gen(seed)
    T, M = B * L, B * L * k + 3
    lens = rows if rows is not None else [L] * B
    used = torch.zeros(T, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        used[b * L: b * L + n] = True
    slot = torch.randperm(M, device="cuda", generator=g)[: T * k].reshape(T, k).int()
    slot[torch.rand((T, k), device="cuda", generator=g) < 0.1] = -1
    slot[T // 2] = -1                                # a token that no expert took
    Y = torch.full((M, D), math.nan, device="cuda", dtype=torch.bfloat16)
    live = slot[used]
    live = live[live >= 0].long()
    Y[live] = bf16(randn(g, live.numel(), D))        # no other row may be read
    gate = torch.rand((T, k), device="cuda", generator=g)
    gate[slot < 0] = math.nan
    res = bf16(randn(g, T, D))
    res[~used] = math.nan
    return dict(T=T, M=M, used=used, slot=slot, Y=Y, gate=gate, res=res, gamma=1 + 0.2 * randn(g, D),
                beta=randn(g, D), dout=bf16(randn(g, T, D)), dsum=bf16(randn(g, T, D)),
                rows=None if rows is None else torch.tensor(rows, dtype=torch.int32, device="cuda"))


def combine_ref(c, gated, scale, res):
    """S in 64 bits, the sum of magnitudes behind it, and the picked rows."""
    s = torch.zeros(c["T"], c["Y"].shape[1], dtype=torch.float64, device="cuda")
    mag, picked = s.clone(), []
    if res:
        s = scale * torch.where(c["used"][:, None], c["res"].double(), 0.0)
        mag = s.abs()
    for j in range(c["slot"].shape[1]):
        ok = (c["slot"][:, j] >= 0) & c["used"]
        y = torch.zeros_like(s)
        y[ok] = c["Y"][c["slot"][ok, j].long()].double()
        gj = torch.where(ok, c["gate"][:, j].double() if gated else 1.0, 0.0)[:, None]
        picked.append((ok, y, gj))
        s, mag = s + gj * y, mag + (gj * y).abs()
    return s, mag, picked


COMBINE = [
    (1, 1, 8, 1, None), (1, 1, 768, 2, None), (2, 9, 64, 2, [9, 4]), (3, 33, 136, 3, [0, 33, 1]),
    (1, 70, 1024, 8, None), (2, 40, 1032, 4, [40, 39]), (1, 5, 8192, 2, None), (4, 500, 768, 2, [500, 1, 0, 321]),
    (1, 3, 8192, 8, None), (1, 700, 520, 3, [699]),
]


@pytest.mark.parametrize("B,L,D,k,rows", COMBINE)
@pytest.mark.parametrize("gated,res,norm,with_sum", [(True, True, True, True), (False, False, False, True),
                                                     (True, False, True, False), (False, True, True, True)])
def test_combine_forward(B, L, D, k, rows, gated, res, norm, with_sum):
    c = combine_inputs(D + k + L, B, L, D, k, rows)
    scale, eps = 0.7, 1e-5
    out = {}
    if with_sum:
        out["sum"] = torch.full((c["T"], D), -5.0, device="cuda", dtype=torch.bfloat16)
    if norm:
        out["out"] = torch.full((c["T"], D), -6.0, device="cuda", dtype=torch.bfloat16)
    sc.expert_combine_forward(c["Y"], c["slot"], c["gate"] if gated else None, B=B, L=L, rows=c["rows"],
                              res=c["res"] if res else None, res_scale=scale,
                              gamma=c["gamma"] if norm else None, beta=c["beta"] if norm else None,
                              eps=eps, out=out)
    scale = float(torch.tensor(scale, dtype=torch.float32))
    s, mag, _ = combine_ref(c, gated, scale, res)
    used = c["used"]
    es = (k + 3) * U_F32 * mag                        # S in fp32
    if with_sum:
        check(out["sum"][used], s[used], es[used], U_BF16, "sum")
        assert bool((out["sum"][~used] == -5.0).all())
    if norm:
        mean = s.mean(dim=1, keepdim=True)
        var = ((s - mean) ** 2).mean(dim=1, keepdim=True)
        inv = 1 / torch.sqrt(var + eps)
        h = (s - mean) * inv
        gam, bet = c["gamma"].double(), c["beta"].double()
        # errors of S, of the mean (of D terms), of 1 / sigma; h is at most sqrt(D)
        d = es.amax(dim=1, keepdim=True) + 16 * U_F32 * (mag.mean(dim=1, keepdim=True) + mean.abs())
        slack = (4 * d * inv * (1 + h.abs()) + 24 * U_F32 * (1 + h.abs())) * gam.abs() + U_F32 * bet.abs()
        check(out["out"][used], (h * gam + bet)[used], slack[used], U_BF16, "out")
        assert bool((out["out"][~used] == -6.0).all())


@pytest.mark.parametrize("B,L,D,k,rows", COMBINE)
@pytest.mark.parametrize("gated,res,norm,dsum", [(True, True, True, True), (False, False, False, True),
                                                 (True, True, True, False)])
def test_combine_backward(B, L, D, k, rows, gated, res, norm, dsum):
    c = combine_inputs(2 * D + k + L, B, L, D, k, rows)
    used = c["used"]
    c["dout"][~used] = math.nan
    c["dsum"][~used] = math.nan
    T, M, scale, eps = c["T"], c["M"], 1.25, 1e-5
    new = lambda *shape, dtype=torch.float32: torch.full(shape, -5.0, device="cuda", dtype=dtype)  # noqa: E731
    out = {"dY": new(M, D, dtype=torch.bfloat16), "dgate": new(T, k)}
    if res:
        out["dres"] = new(T, D, dtype=torch.bfloat16)
    if norm:
        out.update(dgamma=new(D), dbeta=new(D))
    ws = sc.new_expert_workspace(B, L, k, k, D)
    args = dict(B=B, L=L, rows=c["rows"], res=c["res"] if res else None, res_scale=scale, eps=eps,
                gamma=c["gamma"] if norm else None, dout=c["dout"] if norm else None,
                dsum=c["dsum"] if dsum else None, workspace=ws)
    sc.expert_combine_backward(c["Y"], c["slot"], c["gate"] if gated else None, out=out, **args)
    s, mag, picked = combine_ref(c, gated, scale, res)
    mean = s.mean(dim=1, keepdim=True)
    inv = 1 / torch.sqrt(((s - mean) ** 2).mean(dim=1, keepdim=True) + eps)
    h = (s - mean) * inv
    zero = torch.zeros_like(s)
    do = torch.where(used[:, None], c["dout"].double(), 0.0) if norm else zero
    ds = torch.where(used[:, None], c["dsum"].double(), 0.0) if dsum else zero
    eh = torch.zeros_like(s)
    slack = U_F32 * ds.abs()
    if norm:
        d = (k + 3) * U_F32 * mag.amax(dim=1, keepdim=True) + 16 * U_F32 * mag.mean(dim=1, keepdim=True)
        eh = 4 * d * inv * (1 + h.abs()) + 24 * U_F32 * (1 + h.abs())     # of h
        dh = do * c["gamma"].double()
        ab = (dh * h).mean(dim=1, keepdim=True)
        ds = ds + inv * (dh - dh.mean(dim=1, keepdim=True) - h * ab)
        size = dh.abs() + dh.abs().mean(dim=1, keepdim=True) + h.abs() * (dh * h).abs().mean(dim=1, keepdim=True)
        rel = eh.amax(dim=1, keepdim=True) / (1 + h.abs().amax(dim=1, keepdim=True))  # of 1 / sigma, of ab
        slack = slack + inv * (size * (rel + 24 * U_F32) + eh * (ab.abs() + (dh.abs() * eh).mean(dim=1, keepdim=True))
                               + h.abs() * (dh.abs() * eh).mean(dim=1, keepdim=True))
        n = float(used.sum()) + 16
        check(out["dgamma"], (do * h).sum(dim=0),
              (do.abs() * (eh + 2 * U_F32 * h.abs())).sum(dim=0) + n * U_F32 * (do * h).abs().sum(dim=0), 0.0, "dgamma")
        check(out["dbeta"], do.sum(dim=0), n * U_F32 * do.abs().sum(dim=0), 0.0, "dbeta")
    slack = torch.where(used[:, None], slack, 0.0)
    if res:
        check(out["dres"][used], (scale * ds)[used], (2 * scale * slack + U_F32 * ds.abs())[used], U_BF16, "dres")
        assert bool((out["dres"][~used] == -5.0).all())
    touched = torch.zeros(M, dtype=torch.bool, device="cuda")
    for j, (ok, y, gj) in enumerate(picked):
        at = c["slot"][ok, j].long()
        touched[at] = True
        check(out["dY"][at], (gj * ds)[ok], (2 * gj * slack + U_F32 * (gj * ds).abs())[ok], U_BF16, "dY")
        dot, most = (ds * y).sum(dim=1), (ds * y).abs().sum(dim=1)
        check(out["dgate"][:, j], dot, (slack * y.abs()).sum(dim=1) + (D + 16) * U_F32 * most, 0.0, "dgate")
    assert bool((out["dY"][~touched] == -5.0).all())
    again = sc.expert_combine_backward(c["Y"], c["slot"], c["gate"] if gated else None,
                                       out={n: t.clone() for n, t in out.items()}, **args)
    for name in out:
        assert torch.equal(again[name], out[name]), name


@pytest.mark.parametrize("B,L,D,k,rows", [
    (5, 8000, 64, 3, [8000, 1, 7999, 0, 4001]),     # ten rows and more for each warp
    (3, 2100, 1032, 2, [2100, 999, 2]),             # of two warps
    (2, 640, 8192, 8, [640, 633]),                  # one row at a time
])
@pytest.mark.parametrize("gated,res,norm,more", [(True, True, True, True), (False, False, True, False)])
def test_combine_of_many_rows(B, L, D, k, rows, gated, res, norm, more):
    test_combine_forward(B, L, D, k, rows, gated, res, norm, more)
    test_combine_backward(B, L, D, k, rows, gated, res, norm, more)


def test_combine_backward_is_the_difference_quotient():
    """Every gradient of the block's end against central differences of its definition in 64 bits."""
    B, L, D, k, scale, eps, step = 1, 4, 16, 2, 1.25, 1e-5, 1e-5
    c = combine_inputs(77, B, L, D, k, None)
    c["Y"] = bf16(randn(gen(1), c["M"], D))
    c["gate"] = torch.rand((L, k), device="cuda", generator=gen(2))
    got = sc.expert_combine_backward(c["Y"], c["slot"], c["gate"], B=B, L=L, res=c["res"], res_scale=scale,
                                     gamma=c["gamma"], eps=eps, dout=c["dout"], dsum=c["dsum"],
                                     out={"dY": torch.zeros(c["M"], D, device="cuda", dtype=torch.bfloat16),
                                          "dgate": torch.zeros(L, k, device="cuda"),
                                          "dres": torch.zeros(L, D, device="cuda", dtype=torch.bfloat16),
                                          "dgamma": torch.zeros(D, device="cuda"), "dbeta": torch.zeros(D, device="cuda")})
    at = {"dY": c["Y"].double(), "dgate": c["gate"].double(), "dres": c["res"].double(),
          "dgamma": c["gamma"].double(), "dbeta": c["beta"].double()}

    def loss(v):
        s = scale * v["dres"]
        for j in range(k):
            ok = (c["slot"][:, j] >= 0)[:, None]
            s = s + torch.where(ok, v["dgate"][:, j: j + 1] * v["dY"][c["slot"][:, j].clamp(min=0).long()], 0.0)
        o = torch.nn.functional.layer_norm(s, (D,), v["dgamma"], v["dbeta"], eps)
        return (o * c["dout"].double()).sum() + (s * c["dsum"].double()).sum()

    for name in at:
        flat = at[name].reshape(-1)
        for i in range(0, flat.numel(), 1 if flat.numel() < 40 else 5):
            ends = []
            for sign in (1, -1):
                moved = flat.clone()
                moved[i] += sign * step
                ends.append(loss({**at, name: moved.reshape(at[name].shape)}))
            slope = (ends[0] - ends[1]) / (2 * step)
            # bf16 rounding of the gradient, the quotient's own error (1e-16 / step and step^2)
            check(got[name].reshape(-1)[i].cpu(), slope.cpu(), 2e-5,
                  U_BF16 if name in ("dY", "dres") else 1e-6, name)
