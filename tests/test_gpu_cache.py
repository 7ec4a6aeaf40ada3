"""The pruned key-value cache: append, attention with accumulated weights, eviction, and runs of them together,
against plain 64-bit evaluations (``cache_reference``, whose slack is derived there; 2^-25 is half a step of fp16 below 2^-14)."""
import math

import pytest
import torch

import cache_reference as ref
import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
NAN = float("nan")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def strided(t, order):
    """The same values with memory in the order of dimensions given, and room between the slots."""
    if order is None:
        return t
    wide = torch.full([t.shape[i] for i in order[:-1]] + [t.shape[3] + 8], NAN, dtype=t.dtype, device="cuda")
    view = wide.permute([order.index(i) for i in range(3)] + [3])[..., :t.shape[3]]
    view.copy_(t)
    return view


def make_cache(g, B, Hk, C, d, G, lens, dtype=BF, order=None, new=0, evicted=2):
    """lens: slots in use of every sequence (or of each list).  Positions are distinct and in no order, the ``new`` newest ones
    last; what lies behind is NaN."""
    K, V = randn(g, B, Hk, C, d).to(dtype), randn(g, B, Hk, C, d).to(dtype)
    acc = randn(g, B, G, C).abs()
    pos = torch.full((B, G, C), -7, dtype=torch.int32, device="cuda")
    length = torch.tensor([[n] * G if isinstance(n, int) else n for n in lens], dtype=torch.int32, device="cuda")
    seen = i32(*[evicted * max(x) + 5 for x in length.tolist()])
    for b in range(B):
        for i in range(G):
            n = int(length[b, i])
            s = int(seen[b])
            old = torch.randperm(s - new, device="cuda", generator=g)[:max(n - new, 0)]
            pos[b, i, :n] = torch.cat([old, torch.arange(s - new, s, device="cuda")])[:n].int()
            own = slice(i * Hk // G, (i + 1) * Hk // G)
            K[b, own, n:], V[b, own, n:], acc[b, i, n:] = NAN, NAN, NAN
    return dict(K=strided(K, order), V=strided(V, order), acc=acc, pos=pos, len=length, seen=seen)


def copy(cache):
    """As it is, strides too."""
    out = {}
    for n, t in cache.items():
        out[n] = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda")
        out[n].copy_(t)
    return out


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=12345.0), torch.nan_to_num(b.float(), nan=12345.0))


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("B,L,H,Hk,G,d,rot,inter,norm,rows,lens,C,dtype,order", [
    (1, 1, 12, 12, 1, 64, 64, False, True, None, [0], 1, BF, None),
    (1, 1, 12, 12, 1, 64, 64, False, True, None, [100], 128, BF, None),
    (3, 5, 8, 2, 2, 128, 64, True, True, [5, 0, 2], [7, 30, [3, 9]], 40, HF, None),
    (2, 33, 4, 4, 4, 64, 0, False, False, None, [0, [1, 2, 3, 4]], 50, BF, (0, 2, 1, 3)),
    (2, 3, 0, 6, 3, 80, 32, False, True, [1, 3], [10, 11], 15, BF, (1, 0, 2, 3)),
    (1, 2000, 12, 3, 1, 64, 64, False, True, [1999], [77], 2100, BF, None),
    (70, 1, 4, 2, 2, 256, 256, False, True, None, list(range(70)), 71, HF, None),
])
def test_append(B, L, H, Hk, G, d, rot, inter, norm, rows, lens, C, dtype, order):
    g = gen(B + L + C)
    cache = make_cache(g, B, Hk, C, d, G, lens, dtype, order)
    before = copy(cache)
    T = B * L
    qkv = randn(g, T, (H + 2 * Hk) * d).to(dtype)
    Q, K, V = qkv[:, :H * d] if H else None, qkv[:, H * d:(H + Hk) * d], qkv[:, (H + Hk) * d:]
    gq, gk = (1 + 0.3 * randn(g, d), 1 + 0.3 * randn(g, d)) if norm else (None, None)
    freq = sc.rotary_frequencies(rot)[0] if rot else None
    kw = dict(rows=None if rows is None else i32(*rows), freq=freq, interleaved=inter, mscale=1.1, gamma_q=gq if H else None, gamma_k=gk)
    ws = sc.new_cache_workspace(B, C, H, Hk, width=d, lists=G)
    out = sc.cache_append(cache, Q, K, V, L=L, workspace=ws, **kw)
    assert sc.workspace_status(ws) == sc.SC_OK
    assert out["len"] is cache["len"] and out["seen"] is cache["seen"]
    # the keys and queries are those of the rotation at these positions, bit for bit
    pos = (before["seen"][:, None] + torch.arange(L, device="cuda")).int().contiguous()
    turned = sc.rotate_forward(Q, K, width=d, B=B, L=L, pos=pos, **kw)
    for b in range(B):
        m = L if rows is None else rows[b]
        if H:
            assert torch.equal(out["Q"][b * L:b * L + m], turned["Q"][b * L:b * L + m])
        assert int(cache["seen"][b]) == int(before["seen"][b]) + m
        for i in range(G):
            n = int(before["len"][b, i])
            assert int(cache["len"][b, i]) == n + m
            before["acc"][b, i, n:n + m] = 0
            before["pos"][b, i, n:n + m] = pos[b, :m]
            for h in range(i * Hk // G, (i + 1) * Hk // G):
                before["K"][b, h, n:n + m] = turned["K"][b * L:b * L + m, h * d:(h + 1) * d]
                before["V"][b, h, n:n + m] = V[b * L:b * L + m, h * d:(h + 1) * d]
    for n in ("K", "V", "acc", "pos"):
        assert same(cache[n], before[n]), n


def test_append_to_a_full_cache():
    """What does not fit is not stored, and the workspace says so; other sequences are as ever."""
    g = gen(8)
    B, L, Hk, G, C, d = 3, 4, 2, 2, 16, 64
    cache = make_cache(g, B, Hk, C, d, G, [14, [16, 3], 1])
    before = copy(cache)
    K, V = randn(g, B * L, Hk * d).to(BF), randn(g, B * L, Hk * d).to(BF)
    ws = sc.new_cache_workspace(B, C, Hk, Hk, width=d, lists=G)
    sc.cache_append(cache, None, K, V, L=L, workspace=ws)
    assert sc.workspace_status(ws) == sc.SC_ERR_CAPACITY and sc.workspace_status(ws) == sc.SC_OK
    assert cache["len"].tolist() == [[16, 16], [16, 7], [5, 5]]
    assert torch.equal(cache["seen"], before["seen"] + L)
    kv = K.reshape(B, L, Hk, d).transpose(1, 2)
    before["K"][0, :, 14:] = kv[0, :, :2]
    before["K"][1, 1, 3:7] = kv[1, 1]
    before["K"][2, :, 1:5] = kv[2]
    assert same(cache["K"], before["K"])
    with pytest.raises(sc.SparseCoderError):   # (the status code has its text)
        raise sc.SparseCoderError(sc.SC_ERR_CAPACITY, sc.status_string(sc.SC_ERR_CAPACITY))


def test_append_elsewhere_leaves_len():
    g = gen(3)
    cache = make_cache(g, 2, 4, 64, 64, 1, [10, 20])
    K, V = randn(g, 6, 4 * 64).to(BF), randn(g, 6, 4 * 64).to(BF)
    own = dict(len=torch.zeros(2, 1, dtype=torch.int32, device="cuda"), seen=torch.zeros(2, dtype=torch.int32, device="cuda"))
    ws = sc.new_cache_workspace(2, 64, 4, 4)
    for _ in range(3):   # the same slots every time
        sc.cache_append(cache, None, K, V, L=3, out=own, workspace=ws)
    assert own["len"].tolist() == [[13], [23]] and cache["len"].tolist() == [[10], [20]]


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def check_attend(cache, Q, T, rows=None, scale=None, decay=1.0, ws=None, in_place=False):
    B, Hk, C, d = cache["K"].shape
    G, H = cache["acc"].shape[1], Q.shape[1] // d
    lens = [T] * B if rows is None else [min(max(r, 0), T) for r in rows]
    O, acc, o_slack, a_slack = ref.attend(cache, Q, T, lens, scale if scale is not None else 1 / math.sqrt(d), decay)  # noqa: E741
    out = {"O": torch.full((B * T, H * d), 7.0, dtype=Q.dtype, device="cuda")}
    if not in_place:
        out["acc"] = torch.full((B, G, C), 9.0, device="cuda")
    before = copy(cache)
    got = sc.cache_attend(cache, Q, T=T, rows=None if rows is None else i32(*rows), scale=scale, decay=decay, out=out, workspace=ws)
    for n in ("K", "V", "pos", "len", "seen") + (() if in_place else ("acc",)):
        assert same(cache[n], before[n]), n
    u = ref.eps_of(Q.dtype)
    for b in range(B):
        live = slice(b * T, b * T + lens[b])
        off = (got["O"][live].double() - O[live]).abs()
        assert bool((off <= u * O[live].abs() * 1.01 + o_slack[live] + 2.0 ** -25).all()), (b, float(off.max()))
        assert bool((got["O"][b * T + lens[b]:(b + 1) * T] == 7).all())
        for i in range(G):
            n = min(max(int(cache["len"][b, i]), 0), C)
            off = (got["acc"][b, i, :n].double() - acc[b, i, :n]).abs()
            assert bool((off <= a_slack[b, i, :n] + acc[b, i, :n].abs() * 2.0 ** -24).all()), (b, i, float(off.max()))
            rest = got["acc"][b, i, n:]
            assert same(rest, before["acc"][b, i, n:]) if in_place else bool((rest == 9).all())
    return got


ATTEND = [  # B, T, H, Hk, G, d, C, lens, rows, dtype, order
    (1, 1, 12, 12, 1, 64, 1, [1], None, BF, None),
    (1, 1, 12, 12, 12, 64, 300, [257], None, BF, None),
    (3, 1, 8, 2, 1, 128, 100, [100, 0, 63], None, BF, None),
    (3, 1, 8, 2, 2, 64, 97, [[1, 64], [65, 0], 97], None, HF, (0, 2, 1, 3)),
    (2, 1, 32, 1, 1, 128, 513, [512, 129], None, BF, None),        # 32 rows a key head
    (2, 1, 17, 1, 1, 64, 200, [130, 200], None, HF, None),
    (2, 1, 15, 5, 5, 128, 70, [70, 64], [1, 0], BF, (2, 0, 1, 3)),
    (2, 4, 8, 2, 2, 64, 200, [128, 150], [4, 2], BF, None),        # 16 rows a key head
    (2, 5, 6, 2, 1, 64, 200, [128, 150], [3, 5], HF, None),
    (2, 3, 10, 2, 1, 128, 150, [128, 3], [3, 3], BF, None),
    (1, 40, 6, 2, 2, 64, 333, [300], [37], BF, None),              # several tiles of rows
    (2, 64, 2, 2, 1, 128, 256, [64, 256], None, BF, (0, 2, 1, 3)),
    (1, 130, 3, 1, 1, 64, 130, [130], None, HF, None),
    (1, 1, 2, 2, 1, 64, 9000, [8999], None, BF, None),             # many parts of a list
    (1, 2, 4, 1, 1, 128, 5000, [4097], None, BF, None),
    (2, 20, 4, 2, 1, 64, 301, [300, 128], [20, 0], HF, (0, 2, 1, 3)),   # 40 rows a key head, two heads a list
    (3, 9, 30, 5, 5, 64, 35, [35, 9, [10, 35, 0, 9, 12]], None, BF, None),
    (1, 512, 4, 2, 1, 64, 4200, [4100], [500], BF, None),          # scores of more than 32 MB
    (1, 600, 2, 1, 1, 128, 7200, [7150], None, HF, (2, 0, 1, 3)),
    (2, 700, 3, 3, 3, 64, 3000, [[3000, 700, 64], 2990], [700, 3], BF, None),
]


@pytest.mark.parametrize("B,T,H,Hk,G,d,C,lens,rows,dtype,order", ATTEND)
def test_attend(B, T, H, Hk, G, d, C, lens, rows, dtype, order):
    g = gen(T * H + C + d)
    cache = make_cache(g, B, Hk, C, d, G, lens, dtype, order, new=T if all(isinstance(n, int) and n >= T for n in lens) else 0)
    wide = randn(g, B * T, H * d + 16).to(dtype)
    if rows is not None:
        for b, m in enumerate(rows):
            wide[b * T + m:(b + 1) * T] = NAN
    check_attend(cache, wide[:, 8:-8], T, rows, decay=0.75)
    check_attend(cache, wide[:, 8:-8], T, rows, scale=0.3, in_place=True)


def test_attend_many_parts_and_ties():
    """Equal scores everywhere: every weight is 1 / n."""
    for n in (1, 31, 1024, 20011):
        K = torch.ones(1, 2, n, 64, dtype=BF, device="cuda")
        V = torch.ones_like(K)
        cache = dict(K=K, V=V, acc=torch.zeros(1, 1, n, device="cuda"), pos=torch.arange(n, dtype=torch.int32, device="cuda")[None, None].contiguous(),
                     len=i32(n)[None], seen=i32(n))
        out = sc.cache_attend(cache, torch.ones(1, 4 * 64, dtype=BF, device="cuda"), T=1)
        assert bool((out["O"].float() - 1).abs().max() <= 2.0 ** -8)
        assert float((out["acc"] * n - 1).abs().max()) <= 2.0 ** -20


@pytest.mark.parametrize("T,H", [(1, 2), (1, 20), (6, 2), (40, 2)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attend_hidden_slots(T, H, dtype):
    """Slots without a position, or of tokens yet to come, may hold anything; a row that sees none gets 0."""
    g = gen(T)
    cache = make_cache(g, 2, 1, 150, 64, 1, [140, 90], dtype, new=T)
    hide = torch.zeros(2, 1, 150, dtype=torch.bool, device="cuda")
    hide[0, 0, 5:80:3] = True
    hide[0, 0, 64:128] = True            # a whole tile
    hide[1, 0, :90] = True               # a whole list
    cache["pos"][hide] = -1
    cache["pos"][0, 0, 7] = 10 ** 6      # not yet
    hide[0, 0, 7] = True
    for bad in (NAN, math.inf, -math.inf):
        cache["K"][hide.expand(2, 1, 150)] = bad
        cache["V"][hide.expand(2, 1, 150)] = bad
        Q = randn(g, 2 * T, H * 64).to(dtype)
        clean = dict(cache, K=torch.where(hide[..., None], 0, cache["K"]), V=torch.where(hide[..., None], 0, cache["V"]))
        want = sc.cache_attend(clean, Q, T=T, out=dict(acc=cache["acc"].clone(), O=torch.zeros(2 * T, H * 64, dtype=dtype, device="cuda")))
        got = check_attend(cache, Q, T)
        assert torch.equal(got["O"], want["O"])
        assert bool((got["O"][T:] == 0).all()) and bool((got["acc"][1, 0, :90] == cache["acc"][1, 0, :90]).all())


@pytest.mark.parametrize("T", [1, 7, 50])
def test_attend_extreme_scores(T):
    """Scores hundreds apart (one slot has all the weight), all far below zero, and a row of NaN."""
    g = gen(2)
    cache = make_cache(g, 1, 2, 400, 64, 2, [390], BF, new=T)
    cache["K"].mul_(8)
    Q = (8 * randn(g, T, 4 * 64)).to(BF)
    check_attend(cache, Q, T)
    check_attend(cache, Q, T, scale=-1.0)
    check_attend(cache, Q, T, scale=0.0)
    Q[T - 1, :64] = NAN
    out = sc.cache_attend(cache, Q, T=T)["O"]
    assert bool(out[T - 1, :64].isnan().all()) and not bool(out[T - 1, 64:].isnan().any()) and not bool(out[:T - 1].isnan().any())


def test_attend_fp16_small_weights():
    """Many small weights beside a large one keep their digits in fp16."""
    n = 60000
    K = torch.zeros(1, 1, n, 64, dtype=HF, device="cuda")
    K[0, 0, 0, 0] = 160.0                                         # a score of 20: the others weigh e^-20 of it
    V = torch.full((1, 1, n, 64), 1000.0, dtype=HF, device="cuda")
    V[0, 0, 0] = 0
    cache = dict(K=K, V=V, acc=torch.zeros(1, 1, n, device="cuda"), pos=torch.arange(n, dtype=torch.int32, device="cuda")[None, None].contiguous(),
                 len=i32(n)[None], seen=i32(n))
    Q = torch.zeros(1, 64, dtype=HF, device="cuda")
    Q[0, 0] = 1.0
    got = float(sc.cache_attend(cache, Q, T=1)["O"][0, 5])
    want = 1000 * (n - 1) * math.exp(-20) / (1 + (n - 1) * math.exp(-20))
    assert abs(got - want) <= want * 2.0 ** -5   # a weight of 2^-28.9 + 12 is a subnormal of 2^-24 steps: 2^-8 of itself, and sums


def test_attend_long_cache():
    """More than 2^31 elements before the last slot."""
    B, Hk, C, d = 5, 16, 262144, 128
    free, _ = torch.cuda.mem_get_info()
    if free < 30 << 30:
        pytest.skip("needs 30 GB")
    K = torch.zeros(B, Hk, C, d, dtype=BF, device="cuda")
    V = torch.zeros_like(K)
    n = C - 3
    cache = dict(K=K, V=V, acc=torch.zeros(B, 1, C, device="cuda"), pos=torch.arange(C, dtype=torch.int32, device="cuda").repeat(B, 1, 1).contiguous(),
                 len=torch.full((B, 1), n, dtype=torch.int32, device="cuda"), seen=torch.full((B,), C, dtype=torch.int32, device="cuda"))
    Q = torch.zeros(B, Hk * d, dtype=BF, device="cuda")
    Q[:, ::d] = 30.0
    K[B - 1, Hk - 1, n - 1, 0] = 30.0                              # a score of 79 in the last slot alone
    V[B - 1, Hk - 1, n - 1] = 3.0
    V[B - 1, Hk - 1, n:] = NAN
    out = sc.cache_attend(cache, Q, T=1)
    assert bool((out["O"][B - 1, -d:] == 3).all()) and float(out["O"][:, :-d].abs().max()) == 0
    want = (1 + (Hk - 1) / n) / Hk
    assert abs(float(out["acc"][B - 1, 0, n - 1]) - want) <= want * 2.0 ** -19
    # and eviction: that slot comes to the front
    ev = sc.cache_evict(cache, budget=C // 2)
    assert bool((ev["len"] == C // 2).all())
    at = torch.nonzero(ev["pos"][B - 1, 0, :C // 2] == n - 1)
    assert at.shape[0] == 1 and float(K[B - 1, Hk - 1, int(at), 0]) == 30.0 and float(V[B - 1, Hk - 1, int(at), 5]) == 3.0


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------
def check_evict(cache, **kw):
    K, V, acc, pos, length = ref.evict(cache, kw["budget"], kw.get("slack", 0), kw.get("sinks", 0), kw.get("recent", 0))
    apart = copy(cache)
    B, G, C = acc.shape
    out = dict(acc=torch.full((B, G, C), 9.0, device="cuda"), pos=torch.full((B, G, C), 9, dtype=torch.int32, device="cuda"),
               len=torch.zeros(B, G, dtype=torch.int32, device="cuda"))
    sc.cache_evict(apart, out=out, **kw)
    live = torch.arange(C, device="cuda") < length[..., None]
    assert torch.equal(out["len"], length)
    assert same(apart["K"], K) and same(apart["V"], V)
    assert same(torch.where(live, out["acc"], 9), torch.where(live, acc, 9)) and bool((out["acc"][~live] == 9).all())
    assert torch.equal(torch.where(live, out["pos"], 9), torch.where(live, pos, 9)) and bool((out["pos"][~live] == 9).all())
    for n in ("acc", "pos", "len", "seen"):
        assert same(apart[n], cache[n]), n
    sc.cache_evict(cache, **kw)
    for n, t in (("K", K), ("V", V), ("acc", acc), ("pos", pos), ("len", length)):
        assert same(cache[n], t), n


@pytest.mark.parametrize("B,Hk,G,d,C,lens,kw,dtype,order", [
    (1, 12, 1, 64, 8, [1], dict(budget=1), BF, None),
    (1, 12, 1, 64, 8, [2], dict(budget=1), BF, None),
    (1, 12, 1, 64, 100, [0], dict(budget=5), BF, None),
    (2, 4, 4, 128, 300, [[0, 100, 101, 300], 150], dict(budget=100, sinks=4, recent=30), BF, None),
    (2, 4, 2, 64, 1100, [1100, 1025], dict(budget=1024), HF, (0, 2, 1, 3)),
    (2, 4, 2, 64, 1100, [1100, 1030], dict(budget=1024, slack=6), BF, None),
    (2, 4, 2, 64, 1100, [1031, 1030], dict(budget=1024, slack=6), BF, None),
    (1, 3, 3, 80, 5000, [4999], dict(budget=77, sinks=1, recent=76), BF, (1, 0, 2, 3)),
    (1, 2, 1, 256, 5000, [4999], dict(budget=4990), BF, None),
    (3, 1, 1, 16, 40, [40, 39, 3], dict(budget=40), BF, None),
    (3, 1, 1, 16, 40, [40, 39, 3], dict(budget=1000), BF, None),
    (1, 1, 1, 96, 70001, [70000], dict(budget=30000, recent=5000), BF, None),
    (1, 2, 2, 64, 5000, [[5000, 2500]], dict(budget=2500, recent=2500), BF, None),
    (2, 1, 1, 16, 9000, [9000, 33], dict(budget=32), BF, None),                       # two CTAs a list
    (1, 2, 2, 16, 20001, [[20001, 10]], dict(budget=10000, sinks=3, recent=99), HF, None),   # four
    (3, 1, 1, 16, 50003, [50003, 40000, 7], dict(budget=7000, slack=100), BF, None),      # eight
    (200, 1, 1, 16, 8300, [8300 - i for i in range(200)], dict(budget=8200), BF, None),    # too many for more than one
])
def test_evict(B, Hk, G, d, C, lens, kw, dtype, order):
    g = gen(C + d)
    check_evict(make_cache(g, B, Hk, C, d, G, lens, dtype, order), **kw)


@pytest.mark.parametrize("kind", ["equal", "zeros", "coarse", "extremes", "negative", "hidden", "same top bits"])
@pytest.mark.parametrize("n,budget", [(200, 64), (3000, 1500), (3000, 2999), (33000, 20000)])
def test_evict_ranks(kind, n, budget):
    g = gen(n + budget)
    cache = make_cache(g, 2, 2, n + 3, 64, 2, [n, n - 7])
    acc = cache["acc"]
    live = ~acc.isnan()
    if kind == "equal":
        acc[live] = 0.25
    elif kind == "zeros":
        acc.copy_(torch.where(live, torch.where(randn(g, *acc.shape) > 0, 0.0, -0.0), acc))
        acc[:, :, ::50] = 1.0
    elif kind == "coarse":
        acc.copy_((acc * 4).round() / 4)
    elif kind == "extremes":
        pick = torch.randint(0, 8, acc.shape, device="cuda", generator=g)
        top = torch.finfo(torch.float32)
        for i, v in enumerate((NAN, math.inf, -math.inf, top.max, top.min, top.tiny / 4)):
            acc[pick == i] = v
    elif kind == "negative":
        acc.neg_()
    elif kind == "hidden":
        cache["pos"][torch.rand(acc.shape, device="cuda", generator=g) < 0.3] = -1
    else:
        acc.copy_(torch.where(live, 1 + torch.randint(0, 200, acc.shape, device="cuda", generator=g) * 2.0 ** -23, acc))
    check_evict(cache, budget=budget, sinks=3, recent=budget // 4)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("G,Hk,H,d,graph", [(1, 3, 12, 64, False), (2, 2, 2, 128, False), (1, 4, 4, 64, True), (2, 4, 8, 64, True)])
def test_steps(G, Hk, H, d, graph):
    """A prompt, then steps of one or a few tokens with eviction, each step against 64 bits from the same state: the
    cache in 64 bits goes on from the kernels' own rounded values, so that a slot near the cut is the same for both."""
    g = gen(G + H)
    B, C, T, budget = 3, 96, 4, 48
    cache = sc.new_cache(B, C, Hk, width=d, lists=G)
    ws = sc.new_cache_workspace(B, C, H, Hk, width=d, lists=G, T=40)
    freq, gamma = sc.rotary_frequencies(d)[0], 1 + 0.2 * randn(g, d)
    kw = dict(freq=freq, gamma_q=gamma, gamma_k=gamma, workspace=ws)
    qkv = lambda n: [randn(g, n, h * d).to(BF) for h in (H, Hk, Hk)]  # noqa: E731
    # the prompt: ragged, the last rows of it score the slots
    rows = [40, 7, 0]
    Q, K, V = qkv(B * 40)
    q = sc.cache_append(cache, Q, K, V, L=40, rows=i32(*rows), **kw)["Q"]
    check_attend(cache, q, 40, rows, ws=ws, in_place=True)
    check_evict(cache, budget=budget, sinks=2, recent=8)
    Q, K, V = qkv(B * T)
    r = i32(*[T] * B)
    out = {"Q": torch.zeros_like(Q)}
    att = {"O": torch.zeros_like(Q)}

    def step():
        sc.cache_append(cache, Q, K, V, L=T, rows=r, out=out, **kw)
        sc.cache_attend(cache, out["Q"], T=T, rows=r, decay=0.9, out=att, workspace=ws)
        sc.cache_evict(cache, budget=budget, slack=7, sinks=2, recent=8, workspace=ws)

    captured = None
    if graph:
        kept = copy(cache)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        assert all(same(cache[n], kept[n]) for n in cache)   # nothing ran yet
    for i in range(30):
        for t, new in zip((Q, K, V), qkv(B * T)):
            t.copy_(new)
        rows = [1 + i % T, (i * 7) % (T + 1), T if i % 3 else 0]
        r.copy_(i32(*rows))
        plain = copy(cache)
        captured.replay() if graph else step()
        sc.cache_append(plain, Q, K, V, L=T, rows=r, out={"Q": torch.zeros_like(Q)}, **kw)
        pq = out["Q"]
        O, acc, o_slack, a_slack = ref.attend(plain, pq, T, rows, 1 / math.sqrt(d), 0.9)  # noqa: E741
        u = ref.eps_of(BF)
        for b in range(B):
            live = slice(b * T, b * T + rows[b])
            assert bool(((att["O"][live].double() - O[live]).abs() <= u * O[live].abs() * 1.01 + o_slack[live]).all())
        mine = sc.cache_attend(plain, pq, T=T, rows=r, decay=0.9, workspace=ws)["acc"]
        for b in range(B):
            for j in range(G):
                n = int(plain["len"][b, j])
                assert bool(((mine[b, j, :n].double() - acc[b, j, :n]).abs() <= a_slack[b, j, :n] + 2.0 ** -24 * acc[b, j, :n]).all())
        K2, V2, acc2, pos2, len2 = ref.evict(plain, budget, 7, 2, 8)
        assert torch.equal(cache["len"], len2)
        for b in range(B):
            for j in range(G):
                n = int(len2[b, j])
                assert torch.equal(cache["pos"][b, j, :n], pos2[b, j, :n]) and torch.equal(cache["acc"][b, j, :n], acc2[b, j, :n])
                own = slice(j * Hk // G, (j + 1) * Hk // G)
                assert torch.equal(cache["K"][b, own, :n], K2[b, own, :n]) and torch.equal(cache["V"][b, own, :n], V2[b, own, :n])
    assert sc.workspace_status(ws) == sc.SC_OK
    assert int(cache["len"].max()) <= budget + 7 + T


def test_lengths_out_of_range():
    """len and rows are held within the cache and the call on the device."""
    g = gen(44)
    cache = make_cache(g, 3, 2, 40, 64, 1, [40, 0, 20])
    cache["len"][0, 0], cache["len"][1, 0] = 1000, -5
    for T, rows in ((1, [5, 1, -3]), (3, [3, 2, 100]), (25, [25, 26, 1])):
        check_attend(cache, randn(g, 3 * T, 4 * 64).to(BF), T, rows)
    check_evict(copy(cache), budget=30)
    held = copy(cache)
    K, V = randn(g, 6, 128).to(BF), randn(g, 6, 128).to(BF)
    ws = sc.new_cache_workspace(3, 40, 2, 2)
    sc.cache_append(cache, None, K, V, L=2, rows=i32(1, 7, -1), workspace=ws)
    assert cache["len"].tolist() == [[40], [2], [20]] and (cache["seen"] - held["seen"]).tolist() == [1, 2, 0]
    assert sc.workspace_status(ws) == sc.SC_ERR_CAPACITY
    held["K"][1, :, :2] = K[2:4].reshape(2, 2, 64).transpose(0, 1)
    assert same(cache["K"], held["K"])


def test_one_workspace_for_caches_of_different_sizes():
    """Calls of one stream share a workspace, whatever the sizes of each."""
    g = gen(45)
    caches = [make_cache(g, 2, 4, 700, 64, 4, [650, 700], new=1), make_cache(g, 1, 2, 3000, 128, 1, [2999], HF, new=1)]
    size = max(sc.cache_workspace_size(2, 702, 8, 4, lists=4, T=70), sc.cache_workspace_size(1, 3001, 16, 2, width=128, T=70))
    raw = torch.zeros(size + 256, dtype=torch.uint8, device="cuda")
    ws = raw[-raw.data_ptr() % 256:][:size]
    for i in range(3):
        for c, H in zip(caches, (8, 16)):
            B, Hk, C, d = c["K"].shape
            for T in (1, 40, 70):
                check_attend(c, randn(g, B * T, H * d).to(c["K"].dtype), T, ws=ws, decay=0.5, in_place=True)
            out = sc.cache_evict(c, budget=C - 100 - i, workspace=ws)
            sc.cache_append(c, None, randn(g, B * 2, Hk * d).to(c["K"].dtype), randn(g, B * 2, Hk * d).to(c["K"].dtype), L=2, workspace=ws)
            assert int(out["len"].min()) >= 2 and int(c["len"].max()) == C - 98 - i
    assert sc.workspace_status(ws) == sc.SC_OK


def test_matches_the_whole_sequence_layer():
    """One head, everything seen by the last token: its weights are the rows that the framework's layer
    accumulates, when that token is global and the window covers nothing else."""
    g = gen(1)
    L, H = 40, 2
    q, k, v = (randn(g, 1, L, H, 64).to(BF) for _ in range(3))
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[None]
    O, scores, _, _ = sc.layer_forward(q, k, v, i32(L), pos, L, [], 0.0)   # full attention
    cache = dict(K=k.transpose(1, 2).contiguous(), V=v.transpose(1, 2).contiguous(), acc=torch.zeros(1, 1, L, device="cuda"),
                 pos=torch.zeros(1, 1, L, dtype=torch.int32, device="cuda"), len=i32(L)[None], seen=i32(L))   # (every row sees every slot)
    out = sc.cache_attend(cache, q.reshape(L, H * 64), T=L)
    assert float((out["acc"][0, 0] / L - scores[0]).abs().max()) <= 2e-5   # two bars of 1e-5
    assert float((out["O"].float() - O.reshape(L, H * 64).float()).abs().max()) <= 2 * 2e-2


def test_on_another_stream():
    g = gen(6)
    cache = make_cache(g, 2, 4, 300, 64, 2, [290, 280], new=1)
    Q = randn(g, 2, 8 * 64).to(BF)
    K, V = randn(g, 2, 4 * 64).to(BF), randn(g, 2, 4 * 64).to(BF)
    res = []
    for side in (None, torch.cuda.Stream()):
        c = copy(cache)
        if side is not None:
            side.wait_stream(torch.cuda.current_stream())
        a = sc.cache_append(c, Q, K, V, L=1, stream=side)
        o = sc.cache_attend(c, a["Q"], T=1, stream=side)
        sc.cache_evict(c, budget=200, stream=side)
        (side or torch.cuda.current_stream()).synchronize()
        res.append((o["O"], c))
    assert torch.equal(res[0][0], res[1][0])
    assert all(same(res[0][1][n], res[1][1][n]) for n in cache)


def test_two_streams_at_once():
    """Calls that overlap, with a workspace each."""
    g = gen(16)
    caches = [make_cache(g, 4, 4, 4000, 128, 1, [4000, 3900, 10, 2000], new=1) for _ in range(2)]
    Q = randn(g, 4, 16 * 128).to(BF)
    want = [sc.cache_attend(copy(c), Q, T=1) for c in caches]
    work = [(copy(c), sc.new_cache_workspace(4, 4000, 16, 4, width=128), torch.cuda.Stream()) for c in caches]
    torch.cuda.synchronize()
    for _ in range(20):
        outs = [dict(acc=torch.zeros(4, 1, 4000, device="cuda"), O=torch.zeros_like(Q)) for _ in work]
        torch.cuda.synchronize()
        got = [sc.cache_attend(c, Q, T=1, out=o, workspace=w, stream=s) for (c, w, s), o in zip(work, outs)]
        torch.cuda.synchronize()
        for a, b, c in zip(got, want, caches):
            assert torch.equal(a["O"], b["O"])
            for i, n in enumerate(c["len"][:, 0].tolist()):
                assert torch.equal(a["acc"][i, 0, :n], b["acc"][i, 0, :n])


def test_two_calls_give_the_same_bits():
    g = gen(26)
    for T in (1, 20):
        cache = make_cache(g, 2, 4, 3000, 64, 1, [3000, 2900], new=T)
        Q = randn(g, 2 * T, 8 * 64).to(BF)
        a, b = (sc.cache_attend(copy(cache), Q, T=T) for _ in range(2))
        assert torch.equal(a["O"], b["O"]) and same(a["acc"], b["acc"])


def test_two_graphs_share_a_workspace():
    """Steps of two caches in a graph each, with one workspace, replayed in turn: bit for bit the eager steps with a
    workspace each."""
    g = gen(46)
    shapes = [(2, 4, 300, 64, 4, 8, 1, BF), (1, 2, 2100, 128, 1, 8, 6, HF)]   # B, Hk, C, d, G, H, T, type
    ws = torch.zeros(256 + max(sc.cache_workspace_size(B, C, H, Hk, lists=G, width=d, T=T) for B, Hk, C, d, G, H, T, _ in shapes),
                     dtype=torch.uint8, device="cuda")
    ws = ws[-ws.data_ptr() % 256:]
    sides = []
    for B, Hk, C, d, G, H, T, dt in shapes:
        cache = make_cache(g, B, Hk, C, d, G, [C - 2 * T] * B, dt)
        cache = {n: t.clone() for n, t in cache.items()}
        ins = [randn(g, B * T, h * d).to(dt) for h in (H, Hk, Hk)]
        freq, budget = sc.rotary_frequencies(d)[0], C - 2 * T - 20

        def step(c, w, ins=ins, T=T, freq=freq, budget=budget):
            q = sc.cache_append(c, *ins, L=T, freq=freq, workspace=w)["Q"]
            O = sc.cache_attend(c, q, T=T, decay=0.9, workspace=w)["O"]  # noqa: E741
            sc.cache_evict(c, budget=budget, slack=15, sinks=1, recent=4, workspace=w)
            return O

        mine = {n: t.clone() for n, t in cache.items()}
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            O = step(mine, ws)  # noqa: E741
        own = sc.new_cache_workspace(B, C, H, Hk, lists=G, width=d, T=T)
        sides.append((cache, mine, ins, captured, O, step, own))
    for i in range(12):
        for cache, mine, ins, captured, O, step, own in sides:
            for t in ins:
                t.copy_(randn(g, *t.shape).to(t.dtype))
            captured.replay()
            want = step(cache, own)
            assert torch.equal(O, want), i
            for n in cache:
                assert same(mine[n], cache[n]), (i, n)
    assert sc.workspace_status(ws) == sc.SC_OK
