"""What the operators of a pruned key-value cache are measured on.

The incremental form of the framework's attention with token pruning: tokens come one or a few at a time, their keys and
values go into a cache, every step's attention adds its weights to the slots that it read, and the slots with the least
accumulated weight are evicted.  Five kinds of case, each one public call:

  rotate        ``rotate_forward``: norm of each query and key head, and the rotation by position
  rotate_back   ``rotate_backward``
  append        ``cache_append``: the same pass, keys and values into the cache
  attend        ``cache_attend``: attention over the cache, its weights accumulated per slot
  evict         ``cache_evict``: the slots to keep, and the rows that move

A cache has ``G`` lists of slots a sequence; a list has ``Hk / G`` of the key-value heads, which keep and drop slots together:
K, V [B, Hk, C, d], acc and pos [B, G, C], len [B, G], seen [B] (positions given out so far).  Slots come in no
particular order: ``pos`` says which token a slot holds.  What a call leaves untouched (rows and slots past the ones in
use) is zero in every output, because the outputs are cleared once beforehand.
"""
from __future__ import annotations

import math

import torch

own = False   # False: plain elementary operations in 32 bits; True: the framework's operators

EPS = 1e-6


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _case(name, kind, B, L, H, Hk, d, *, C=0, G=1, fill=1.0, ragged=1.0, rot=0, inter=False, norm=False, far=0, mscale=1.0,
          half=False, budget=0, slack=0, sinks=0, recent=0, decay=1.0):
    """L tokens a sequence come with the call (``ragged``: rows in use uniform in [ragged L, L]).  Lists hold ``fill`` C
    slots, or, where ``ragged`` < 1 and L is 1, between ragged fill C and fill C.  Positions start at ``far``.  ``half``:
    fp16 in place of bf16."""
    return dict(name=name, kind=kind, B=B, L=L, H=H, Hk=Hk, d=d, C=C, G=G, fill=fill, ragged=ragged, rot=rot, inter=inter,
                norm=norm, far=far, mscale=mscale, half=half, budget=budget, slack=slack, sinks=sinks, recent=recent,
                decay=decay)


def listed():
    return [
        # a training batch of functions after token pruning: ragged rows, queries and keys normalised
        _case("rotate_1024", "rotate", 8, 1024, 12, 12, 64, rot=64, norm=True, ragged=0.6),
        # the longest inputs far into a long document, half of the head rotated, neighbouring features paired
        _case("rotate_4096_part", "rotate", 4, 4096, 16, 4, 128, rot=64, inter=True, far=1_000_000, mscale=1.25),
        # gradients of an ordinary batch
        _case("rotate_back_512", "rotate_back", 4, 512, 16, 16, 64, rot=64, norm=True),
        # ... and of the longest inputs: the largest of its kind
        _case("rotate_back_4096", "rotate_back", 4, 4096, 16, 4, 128, rot=128, norm=True),
        # one token of one stream goes into the cache: latency only
        _case("append_one", "append", 1, 1, 12, 12, 64, C=4096, fill=0.5, rot=64, norm=True),
        # the prompts of a batch, one list of slots for each key-value head
        _case("append_prompt", "append", 4, 4096, 12, 4, 64, C=8192, G=4, fill=0.25, ragged=0.8, rot=64, norm=True, far=100_000),
        # one token of one stream: a scanner that reads code as it is typed
        _case("attend_one", "attend", 1, 1, 12, 12, 64, C=2048, fill=0.5),
        # a serving batch, streams of different lengths
        _case("attend_batch", "attend", 32, 1, 16, 4, 128, C=8192, ragged=0.4),
        # one very long stream with two lists
        _case("attend_long", "attend", 1, 1, 16, 2, 128, C=131072, G=2, fill=0.99, decay=0.999),
        # the last tokens of the prompts score the slots before the first eviction, each head for itself
        _case("attend_window", "attend", 4, 32, 12, 12, 64, C=4096, G=12),
        # one stream is brought back to its budget
        _case("evict_one", "evict", 1, 1, 12, 12, 64, C=2048, fill=0.55, budget=1024, sinks=4, recent=64),
        # a batch after its prompts, half of the slots go, each head for itself
        _case("evict_batch", "evict", 32, 1, 16, 4, 128, C=8192, G=4, budget=4096, sinks=4, recent=256, ragged=0.9),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "rotate_back", "append", "append", "attend", "attend", "attend", "attend", "evict", "evict"])
    d = rng.choice([64, 64, 128])
    Hk = rng.choice([1, 2, 4, 5, 8, 12, 16])
    H = Hk * rng.choice([1, 1, 2, 3, 4, 8])
    while H > 32:
        H -= Hk
    G = rng.choice([1, 1, Hk])
    c = dict(norm=rng.random() < 0.6, half=rng.random() < 0.25, rot=rng.choice([d, d, d // 2, 16]), inter=rng.random() < 0.4,
             far=rng.choice([0, 0, 5000, 2_000_000]), mscale=rng.choice([1.0, 1.0, 1.1]), ragged=rng.choice([1.0, 1.0, 0.5, 0.8]))
    if kind in ("rotate", "rotate_back", "append"):
        L = _log_uniform(rng, 1, 4096)
        B = max(1, min(64, _log_uniform(rng, L, 16384) // L))
        while B * L * (H + 2 * Hk) * d > 16384 * 24 * 128:
            L, B = max(1, L // 2), max(1, B - 1)
        if kind == "append":
            C = L + _log_uniform(rng, 1, 4096)
            c.update(C=C, G=G, fill=rng.uniform(0, 1) * (C - L) / C)
        return _drawn(kind, B, L, H, Hk, d, c)
    C = _log_uniform(rng, 16, 65536)
    B = max(1, min(64, _log_uniform(rng, C, 262144) // C))
    L = 1
    if kind == "attend" and rng.random() < 0.4:
        L = min(_log_uniform(rng, 1, 64), C)
    while B * C * Hk * d > 32 * 8192 * 4 * 128 or L * H * B * C > 4 * 32 * 12 * 4096 * 4:
        B, C = max(1, B - 1), max(L, C // 2)
    c.update(C=C, G=G, fill=max(rng.uniform(0.2, 1.0), L / C), decay=rng.choice([1.0, 1.0, 0.99]))
    if L > 1:
        c["ragged"] = 1.0
    if kind == "evict":
        n = max(1, int(c["fill"] * C))
        c["budget"] = max(1, int(n * rng.uniform(0.3, 1.0)))
        c["slack"] = rng.choice([0, 0, c["budget"] // 16])
        c["sinks"] = rng.choice([0, 4]) if c["budget"] >= 8 else 0
        c["recent"] = rng.choice([0, c["budget"] // 8, c["budget"] // 2])
    return _drawn(kind, B, L, H, Hk, d, c)


def _drawn(kind, B, L, H, Hk, d, c):
    c = _case("", kind, B, L, H, Hk, d, **c)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    c, kind = case, case["kind"]
    B, L, H, Hk, d, C, G = c["B"], c["L"], c["H"], c["Hk"], c["d"], c["C"], c["G"]
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(1_000_003 * int(seed) + 29)
    low = torch.float16 if c["half"] else torch.bfloat16
    randn = lambda *shape: torch.randn(shape, device=dev, generator=gen)  # noqa: E731
    rand = lambda *shape: torch.rand(shape, device=dev, generator=gen)  # noqa: E731
    zeros = lambda *shape, dtype=low: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    i32 = torch.int32
    st = dict(case=c, rows=None, low=low)
    if c["ragged"] < 1 and L > 1:
        st["rows"] = torch.randint(max(1, int(c["ragged"] * L)), L + 1, (B,), device=dev, generator=gen).int()
    if kind in ("rotate", "rotate_back", "append"):
        # one projection's output holds queries, keys and values side by side; a trained model's heads differ in size
        qkv = (randn(B * L, H + 2 * Hk, d) * (0.5 + rand(H + 2 * Hk, 1))).to(low).reshape(B * L, -1)
        st.update(Q=qkv[:, :H * d], K=qkv[:, H * d:(H + Hk) * d], V=qkv[:, (H + Hk) * d:])
        rot = c["rot"]
        st["freq"] = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot) if rot else None
        st["gamma_q"] = 1 + 0.1 * randn(d) if c["norm"] else None
        st["gamma_k"] = 1 + 0.1 * randn(d) if c["norm"] else None
    if kind in ("rotate", "rotate_back"):
        # positions of the tokens that earlier layers kept: in order, with gaps
        gaps = 1 + (rand(B, L) < 0.3).int()
        st["pos"] = (c["far"] + gaps.cumsum(1) - 1).to(i32)
        if kind == "rotate":
            st["out"] = dict(Q=zeros(B * L, H * d), K=zeros(B * L, Hk * d))
        else:
            st.update(dQ=randn(B * L, H * d).to(low), dK=randn(B * L, Hk * d).to(low))
            st["out"] = dict(dQ=zeros(B * L, H * d), dK=zeros(B * L, Hk * d))
            if c["norm"]:
                st["out"].update(dgamma_q=zeros(d, dtype=torch.float32), dgamma_k=zeros(d, dtype=torch.float32))
        return st
    # the cache: slots in use and the positions that they hold, in no order but that the newest tokens lie last
    new = 0 if kind == "append" else L
    n = torch.full((B,), int(c["fill"] * C), device=dev, dtype=torch.int64)
    if c["ragged"] < 1 and L == 1:
        n = (n * (c["ragged"] + (1 - c["ragged"]) * rand(B))).long()
    n = n.clamp(min=max(new, 1) if kind != "append" else 0, max=C - (L if kind == "append" else 0))
    seen = c["far"] + n + (n * rand(B)).long()                       # some were evicted before
    j = torch.arange(C, device=dev).expand(B, G, C)
    old = (n - new)[:, None, None]
    span = (seen - new)[:, None, None]
    spread = torch.where(j < old, (j * span) // old.clamp(min=1), j - old + span)   # distinct, below seen
    order = torch.argsort(torch.where(j < old, rand(B, G, C), 2.0 + j), dim=2)
    held = j < n[:, None, None]
    pos = torch.where(held, spread.gather(2, order), 0)
    # weights, a step's being 1 / n in the mean: a few tokens hold most of them; the ones that came last have had none yet
    acc = torch.where(held & (j < old), torch.exp(randn(B, G, C) - 0.5), 0.0) / n.clamp(min=1)[:, None, None]
    st["cache"] = dict(K=randn(B, Hk, C, d).to(low), V=randn(B, Hk, C, d).to(low), acc=acc, pos=pos.to(i32),
                       len=n[:, None].expand(B, G).contiguous().to(i32), seen=seen.to(i32))
    if kind == "append":
        st["out"] = dict(Q=zeros(B * L, H * d), len=zeros(B, G, dtype=i32), seen=zeros(B, dtype=i32))
    elif kind == "attend":
        st["Q"] = (1.5 * randn(B * L, H * d)).to(low)
        st["out"] = dict(O=zeros(B * L, H * d), acc=zeros(B, G, C, dtype=torch.float32))
    else:
        st["out"] = dict(acc=zeros(B, G, C, dtype=torch.float32), pos=zeros(B, G, C, dtype=i32), len=zeros(B, G, dtype=i32))
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2310_07109_gb300 as sc
    c, kind, out = st["case"], st["case"]["kind"], st["out"]
    if "ws" not in st:   # the workspace that a program keeps
        st["ws"] = (sc.new_rotate_workspace(c["d"]) if kind.startswith("rotate") else
                    sc.new_cache_workspace(c["B"], c["C"], c["H"], c["Hk"], width=c["d"], lists=c["G"], T=c["L"]))
    turn = dict(rows=st["rows"], L=c["L"])
    if kind != "attend" and kind != "evict":
        turn.update(freq=st["freq"], interleaved=c["inter"], mscale=c["mscale"], gamma_q=st["gamma_q"], gamma_k=st["gamma_k"], eps=EPS)
    if kind == "rotate":
        return sc.rotate_forward(st["Q"], st["K"], width=c["d"], B=c["B"], pos=st["pos"], out=out, **turn)
    if kind == "rotate_back":
        return sc.rotate_backward(st["dQ"], st["dK"], st["Q"], st["K"], width=c["d"], B=c["B"], pos=st["pos"], out=out,
                                  workspace=st["ws"], **turn)
    cache = st["cache"]
    if kind == "append":
        sc.cache_append(cache, st["Q"], st["K"], st["V"], out=out, workspace=st["ws"], **turn)
        return dict(out, K=cache["K"], V=cache["V"], acc=cache["acc"], pos=cache["pos"])
    if kind == "attend":
        return sc.cache_attend(cache, st["Q"], T=c["L"], rows=st["rows"], decay=c["decay"], out=out, workspace=st["ws"])
    sc.cache_evict(cache, budget=c["budget"], slack=c["slack"], sinks=c["sinks"], recent=c["recent"], out=out, workspace=st["ws"])
    return dict(out, K=cache["K"], V=cache["V"])


def _here(st):
    """[B, L]: whether a row is in use."""
    c = st["case"]
    r = torch.arange(c["L"], device="cuda")[None, :]
    return r < (st["rows"][:, None] if st["rows"] is not None else c["L"])


def _angles(st, pos):
    """cos and sin [B, L, 1, rot / 2], scaled; the angles in 64 bits: positions are far."""
    t = pos[..., None].double() * st["freq"]
    m = st["case"]["mscale"]
    return (m * torch.cos(t)).float()[:, :, None], (m * torch.sin(t)).float()[:, :, None]


def _halves(x, rot, inter):
    """The two features of each rotated pair."""
    r = x[..., :rot]
    return (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])


def _joined(a, b, x, rot, inter):
    r = torch.stack((a, b), dim=-1).flatten(-2) if inter else torch.cat((a, b), dim=-1)
    return torch.cat((r, x[..., rot:]), dim=-1)


def _turned(st, x, heads, gamma, pos):
    """Norm and rotation of x [B * L, heads * d]: [B, L, heads, d] in 32 bits."""
    c = st["case"]
    x = x.float().reshape(c["B"], c["L"], heads, c["d"])
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * gamma
    cos, sin = _angles(st, pos)
    a, b = _halves(x, c["rot"], c["inter"])
    return _joined(a * cos - b * sin, b * cos + a * sin, x, c["rot"], c["inter"])


def _turned_back(st, dy, x, heads, gamma, pos, here):
    c = st["case"]
    dy = dy.float().reshape(c["B"], c["L"], heads, c["d"])
    cos, sin = _angles(st, pos)
    a, b = _halves(dy, c["rot"], c["inter"])
    dy = _joined(a * cos + b * sin, b * cos - a * sin, dy, c["rot"], c["inter"])
    if gamma is None:
        return dy, None
    x = x.float().reshape(c["B"], c["L"], heads, c["d"])
    inv = 1 / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    hat = x * inv
    dgamma = torch.where(here, dy * hat, 0.0).sum(dim=(0, 1, 2))
    dh = dy * gamma
    return inv * (dh - hat * (dh * hat).mean(dim=-1, keepdim=True)), dgamma


def _run_plain(st):
    c, kind, low = st["case"], st["case"]["kind"], st["low"]
    B, L, H, Hk, d, C, G = c["B"], c["L"], c["H"], c["Hk"], c["d"], c["C"], c["G"]
    if kind in ("rotate", "rotate_back", "append"):
        here = _here(st).expand(B, L)[:, :, None, None]
        flat = lambda t: torch.where(here, t, 0.0).to(low).reshape(B * L, -1)  # noqa: E731
    if kind == "rotate":
        return dict(Q=flat(_turned(st, st["Q"], H, st["gamma_q"], st["pos"])),
                    K=flat(_turned(st, st["K"], Hk, st["gamma_k"], st["pos"])))
    if kind == "rotate_back":
        dq, gq = _turned_back(st, st["dQ"], st["Q"], H, st["gamma_q"], st["pos"], here)
        dk, gk = _turned_back(st, st["dK"], st["K"], Hk, st["gamma_k"], st["pos"], here)
        out = dict(dQ=flat(dq), dK=flat(dk))
        return dict(out, dgamma_q=gq, dgamma_k=gk) if c["norm"] else out
    k = st["cache"]
    if kind == "append":
        r = torch.arange(L, device="cuda")
        at = k["seen"][:, None] + r
        q, key = _turned(st, st["Q"], H, st["gamma_q"], at), _turned(st, st["K"], Hk, st["gamma_k"], at)
        slot = k["len"].long()[:, :, None] + r                                        # [B, G, L]
        wide = slot.repeat_interleave(Hk // G, dim=1)                                 # [B, Hk, L]
        b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(Hk, device="cuda")[None, :, None]
        for name, t in (("K", key.to(low)), ("V", st["V"].reshape(B, L, Hk, d))):
            k[name][b, h, wide] = torch.where(here.transpose(1, 2), t.transpose(1, 2), k[name][b, h, wide])
        g = torch.arange(G, device="cuda")[None, :, None]
        inside = here[:, None, :, 0, 0]
        k["acc"][b, g, slot] = torch.where(inside, 0.0, k["acc"][b, g, slot])
        k["pos"][b, g, slot] = torch.where(inside, at[:, None, :], k["pos"][b, g, slot]).int()
        come = st["rows"] if st["rows"] is not None else L
        return dict(Q=flat(q), len=k["len"] + (come[:, None] if st["rows"] is not None else L), seen=k["seen"] + come,
                    K=k["K"], V=k["V"], acc=k["acc"], pos=k["pos"])
    j = torch.arange(C, device="cuda")
    held = j < k["len"][:, :, None]                                                   # [B, G, C]
    if kind == "attend":
        R, share = H // Hk, H // G
        q = st["Q"].float().reshape(B, L, Hk, R, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, R * L, d)
        s = torch.matmul(q, k["K"].float().transpose(2, 3)).reshape(B, G, share, L, C) / math.sqrt(d)
        at = k["seen"][:, None] - L + torch.arange(L, device="cuda")                  # [B, L]
        sees = (held[:, :, None, :] & (k["pos"][:, :, None, :] <= at[:, None, :, None]))[:, :, None]
        s = torch.where(sees, s, -math.inf)
        p = torch.exp(s - s.amax(dim=-1, keepdim=True))
        p = p / p.sum(dim=-1, keepdim=True)
        v = torch.where(held.repeat_interleave(Hk // G, dim=1)[..., None], k["V"].float(), 0.0)
        o = torch.matmul(p.reshape(B, Hk, R * L, C), v).reshape(B, H, L, d).transpose(1, 2)
        acc = torch.where(held, c["decay"] * k["acc"] + p.sum(dim=(2, 3)) / share, 0.0)
        return dict(O=o.to(low).reshape(B * L, H * d), acc=acc)
    # evict: a stable sort puts the survivors first; the others' places below the budget are filled in order
    n, most = k["len"].long()[:, :, None], c["budget"]
    late = (k["seen"] - c["recent"])[:, None, None]
    rank = torch.where((k["pos"] < c["sinks"]) | (k["pos"] >= late), math.inf, k["acc"])
    order = torch.argsort(torch.where(held, rank, -math.inf), dim=2, descending=True, stable=True)
    full = n > most + c["slack"]
    keep = torch.zeros_like(held).scatter(2, order, (j < most).expand_as(order)) | ~full
    hole, fill = ~keep & (j < most), keep & held & (j >= most) & full
    to = torch.argsort((~hole).int(), dim=2, stable=True)
    come = torch.argsort((~fill).int(), dim=2, stable=True)
    src = j.expand(B, G, C).scatter(2, to, torch.where(j < hole.sum(dim=2, keepdim=True), come, to))
    after = torch.where(full, most, n)
    rows = src.repeat_interleave(Hk // G, dim=1)[..., None].expand(B, Hk, C, d)
    for name in ("K", "V"):
        k[name].copy_(k[name].gather(2, rows))
    return dict(acc=torch.where(j < after, k["acc"].gather(2, src), 0.0), pos=torch.where(j < after, k["pos"].gather(2, src), 0),
                len=after[..., 0].int(), K=k["K"], V=k["V"])


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _rotor(st, pos):
    """exp(i p f) [B, L, 1, rot / 2]."""
    t = pos.double()[..., None] * st["freq"]
    return st["case"]["mscale"] * torch.polar(torch.ones_like(t), t)[:, :, None]


def _head64(st, x, heads, gamma, pos):
    """From the definition, a pair as a complex number."""
    c = st["case"]
    x = x.double().reshape(c["B"], c["L"], heads, c["d"])
    if gamma is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * gamma.double()
    y = x.clone()
    rot, m = c["rot"], c["rot"] // 2
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, m), slice(m, rot))
    z = torch.complex(x[..., first], x[..., second]) * _rotor(st, pos)
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    st = prepare(case, seed)
    c, kind = case, case["kind"]
    B, L, H, Hk, d, C, G = c["B"], c["L"], c["H"], c["Hk"], c["d"], c["C"], c["G"]
    lens = [L] * B if st["rows"] is None else st["rows"].tolist()
    used = torch.zeros(B, L, dtype=torch.float64, device="cuda")
    for b, m in enumerate(lens):
        used[b, :m] = 1
    if kind == "rotate":
        return {n: (_head64(st, st[n], h, st["gamma_" + n.lower()], st["pos"]) * used[..., None, None]).reshape(B * L, -1)
                for n, h in (("Q", H), ("K", Hk))}
    if kind == "rotate_back":
        out = {}
        for n, h in (("Q", H), ("K", Hk)):
            with torch.enable_grad():
                x = st[n].double().detach().requires_grad_(True)
                g = st["gamma_" + n.lower()]
                g = None if g is None else g.double().requires_grad_(True)
                dy = st["d" + n].double().reshape(B, L, h, d) * used[..., None, None]
                got = torch.autograd.grad(_head64(st, x, h, g, st["pos"]), (x,) if g is None else (x, g), dy)
            out["d" + n] = got[0]
            if g is not None:
                out["dgamma_" + n.lower()] = got[1]
        return out
    cache = {n: (t.double() if t.is_floating_point() else t.long()) for n, t in st["cache"].items()}
    lists = [(b, g, slice(g * Hk // G, (g + 1) * Hk // G), int(cache["len"][b, g])) for b in range(B) for g in range(G)]
    if kind == "append":
        pos = cache["seen"][:, None] + torch.arange(L, device="cuda")
        q = _head64(st, st["Q"], H, st["gamma_q"], pos) * used[..., None, None]
        key, v = _head64(st, st["K"], Hk, st["gamma_k"], pos), st["V"].double().reshape(B, L, Hk, d)
        for b, g, heads, n in lists:
            m = lens[b]
            cache["K"][b, heads, n:n + m] = key[b, :m, heads].transpose(0, 1)
            cache["V"][b, heads, n:n + m] = v[b, :m, heads].transpose(0, 1)
            cache["acc"][b, g, n:n + m] = 0
        return dict(Q=q.reshape(B * L, -1), len=None, seen=None, K=cache["K"], V=cache["V"], acc=cache["acc"], pos=None)
    if kind == "attend":
        O = torch.zeros(B, L, H, d, dtype=torch.float64, device="cuda")  # noqa: E741
        acc = torch.zeros(B, G, C, dtype=torch.float64, device="cuda")
        q, R = st["Q"].double().reshape(B, L, H, d), H // Hk
        for b, g, heads, n in lists:
            acc[b, g, :n] = c["decay"] * cache["acc"][b, g, :n]
            at = int(cache["seen"][b]) - L + torch.arange(L, device="cuda")
            hidden = cache["pos"][b, g, :n][None, :] > at[:, None]
            for h in range(heads.start * R, heads.stop * R):
                s = (q[b, :, h] @ cache["K"][b, h // R, :n].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                p = torch.softmax(s, dim=1)
                O[b, :, h] = p @ cache["V"][b, h // R, :n]
                acc[b, g, :n] += p.sum(dim=0) / (H // G)
        return dict(O=O.reshape(B * L, -1), acc=acc)
    out = torch.zeros(B, G, C, dtype=torch.float64, device="cuda")
    for b, g, heads, n in lists:
        k = n
        if n > c["budget"] + c["slack"]:
            k = c["budget"]
            pos, acc = cache["pos"][b, g, :n].tolist(), cache["acc"][b, g, :n].tolist()
            seen = int(cache["seen"][b])
            order = sorted(range(n), key=lambda i: (not (pos[i] < c["sinks"] or pos[i] >= seen - c["recent"]), -acc[i], i)
                           if not (pos[i] < c["sinks"] or pos[i] >= seen - c["recent"]) else (False, 0.0, i))
            kept = set(order[:k])
            fills = sorted(i for i in kept if i >= k)
            holes = [i for i in range(k) if i not in kept]
            for name in ("K", "V"):
                cache[name][b, heads][:, holes] = cache[name][b, heads][:, fills]
            cache["acc"][b, g, holes] = cache["acc"][b, g, fills]
        out[b, g, :k] = cache["acc"][b, g, :k]
    return dict(acc=out, pos=None, len=None, K=cache["K"], V=cache["V"])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Inputs and outputs once each, at the expected number of rows and slots in use."""
    c, kind = case, case["kind"]
    B, L, H, Hk, d, C, G = c["B"], c["L"], c["H"], c["Hk"], c["d"], c["C"], c["G"]
    mean = (1 + c["ragged"]) / 2
    T = B * L * (mean if L > 1 else 1)
    if kind == "rotate":
        return {"bytes": T * (4 * (H + Hk) * d + 4) + 4 * c["rot"] + 8 * d * c["norm"], "flops": T * (H + Hk) * (3 * c["rot"] + 4 * d * c["norm"])}
    if kind == "rotate_back":
        return {"bytes": T * ((4 + 2 * c["norm"]) * (H + Hk) * d + 4) + 4 * c["rot"] + 16 * d * c["norm"],
                "flops": T * (H + Hk) * (3 * c["rot"] + 12 * d * c["norm"])}
    if kind == "append":
        return {"bytes": T * (4 * (H + 2 * Hk) * d + 8 * G) + 8 * B * (G + 1) + 4 * c["rot"] + 8 * d * c["norm"],
                "flops": T * (H + Hk) * (3 * c["rot"] + 4 * d * c["norm"])}
    n = max(1.0, c["fill"] * C * (mean if L == 1 else 1))
    if kind == "attend":
        return {"bytes": B * n * (4 * Hk * d + 12 * G) + 4 * T * H * d, "flops": 4 * T * H * n * d}
    k = c["budget"]
    if n <= k + c["slack"]:
        return {"bytes": 16.0 * B * G * n, "flops": B * G * n}
    moved = k * (n - k) / n
    return {"bytes": B * (G * (8 * n + 8 * k) + 8 * moved * Hk * d), "flops": B * G * n}
