"""What the expert feed-forward operators are measured on.

A mixture-of-experts feed-forward block on the kept tokens of an encoder layer: a router sends each token to ``k`` of
``E`` experts, every expert's two matrix products run on the rows it was given, and the results are summed under the
router's gates, added to the residual and normalised.  Seven kinds of case, each one public call:

  route           ``expert_route_forward``: the choice, the gates and the expert-sorted slots
  route_back      ``expert_route_backward``
  linear          ``expert_linear_forward``: products grouped by expert (bias, GELU, the value before GELU)
  linear_back_x   ``expert_linear_backward_input``: the gradient of the rows
  linear_back_w   ``expert_linear_backward_weight``: the gradients of the weights and biases
  combine         ``expert_combine_forward``: gated sum, scaled residual, layer norm
  combine_back    ``expert_combine_backward``

Rows of a ragged batch follow the framework's layout: [B][L] with ``rows[b]`` of them in use.  A slot is one (token,
choice) pair in expert order; ``offsets`` [E + 1] bounds each expert's slots.  What a call leaves untouched (rows and
slots past the ones in use) is zero in every output, because the outputs are cleared once beforehand.
"""
from __future__ import annotations

import math

import torch

own = False   # False: plain elementary operations in 32 bits; True: the framework's operators

EPS = 1e-5


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _case(name, kind, B, L, E, k, D=0, F=0, *, ragged=1.0, masked=0.0, coarse=False, renorm=True, gather=False, gelu=False,
          pre=False, f32=False, norm=True, res=True):
    """D -> F is the product of a ``linear`` case (K = D inputs, N = F outputs).  ``ragged``: rows in use per sequence
    uniform in [ragged L, L]; ``masked``: share of the (token, expert) pairs at -inf; ``coarse``: logits rounded to
    bf16, so that ties are frequent."""
    return dict(name=name, kind=kind, B=B, L=L, E=E, k=k, D=D, F=F, ragged=ragged, masked=masked, coarse=coarse,
                renorm=renorm, gather=gather, gelu=gelu, pre=pre, f32=f32, norm=norm, res=res)


def listed():
    return [
        # the router for one token: a streaming scanner that classifies as the user types, latency only
        _case("route_one_token", "route", 1, 1, 8, 2),
        # a batch of functions after token pruning: ragged rows, router computed in bf16 (ties)
        _case("route_1024", "route", 8, 1024, 16, 2, ragged=0.6, coarse=True),
        # fine-grained experts on the longest inputs, a twentieth of the pairs masked (experts out of reach)
        _case("route_4096_e64", "route", 4, 4096, 64, 8, masked=0.05),
        # the router's gradient in training, gates over all experts
        _case("route_back_1024", "route_back", 8, 1024, 64, 4, renorm=False),
        # one token through the first product: two experts' weights are all there is to read
        _case("up_one_token", "linear", 1, 1, 8, 2, 768, 1536, gather=True, gelu=True),
        # one short function (the encoder's smallest ordinary call): a few dozen rows an expert
        _case("up_one_short", "linear", 1, 200, 16, 2, 768, 1536, gather=True, gelu=True),
        # a training batch's first product, the value before GELU kept for the backward pass
        _case("up_1024", "linear", 8, 1024, 8, 2, 768, 1536, gather=True, gelu=True, pre=True),
        # the second product of a wide model on the longest inputs: the largest case
        _case("down_4096", "linear", 4, 4096, 32, 4, 2048, 1024, ragged=0.8),
        # gradient of the hidden rows through the second product, with GELU's derivative
        _case("back_x_1024", "linear_back_x", 8, 1024, 8, 2, 1536, 768, gelu=True),
        # gradient of the first product's weights, rows gathered from the tokens, in 32 bits for the optimizer
        _case("back_w_1024", "linear_back_w", 8, 1024, 8, 2, 768, 1536, gather=True, f32=True),
        # the block's end in a forward pass on ragged rows
        _case("combine_1024", "combine", 8, 1024, 8, 2, 768, ragged=0.6),
        # ... and in training, a wider model with four experts a token
        _case("combine_back_2048", "combine_back", 4, 2048, 32, 4, 1024),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "route_back", "linear", "linear", "linear", "linear_back_x", "linear_back_w", "combine",
                       "combine_back"])
    E = rng.choice([4, 8, 12, 16, 24, 32, 64])
    k = min(E, rng.choice([1, 2, 2, 2, 3, 4, 6, 8]))
    L = _log_uniform(rng, 1, 4096)
    B = max(1, min(32, _log_uniform(rng, L, 16384) // L))
    width = lambda: rng.choice([512, 768, 1024, 1536, 2048, 8 * rng.randint(32, 256)])  # noqa: E731
    D, F = width(), width()
    if kind.startswith("linear"):
        while B * L * k > 65536 or B * L * k * D * F > 65536 * 2048 * 1024 or E * D * F > 32 * 2048 * 1024:
            L, E, k = max(1, L // 2), max(4, E // 2), max(1, k - 1)
    elif kind.startswith("combine"):
        F = 0
    else:
        D = F = 0
    c = _case("", kind, B, L, E, k, D, F, ragged=rng.choice([1.0, 1.0, 0.5, 0.8]),
              masked=rng.choice([0.0, 0.0, 0.05, 0.3]) if kind.startswith("route") else 0.0,
              coarse=kind.startswith("route") and rng.random() < 0.4, renorm=rng.random() < 0.6,
              gather=kind in ("linear", "linear_back_w") and rng.random() < 0.5,
              gelu=kind in ("linear", "linear_back_x") and rng.random() < 0.5,
              f32=kind.startswith("linear") and rng.random() < 0.3, norm=rng.random() < 0.7, res=rng.random() < 0.8)
    c["pre"] = kind == "linear" and c["gelu"] and rng.random() < 0.5
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _route(logits, rows, B, L, k, renorm):
    """The routing in elementary operations: stable sorts give ties to the lowest expert, and slots in expert order
    with the tokens of an expert in their own order."""
    T, E = logits.shape
    dev = logits.device
    here = torch.arange(L, device=dev)[None, :] < (rows[:, None] if rows is not None else L)
    here = here.expand(B, L).reshape(T, 1)
    x = torch.where(here & ~logits.isnan(), logits, -math.inf)
    best, expert = torch.sort(x, dim=1, descending=True, stable=True)
    best, expert = best[:, :k], expert[:, :k]
    chosen = best > -math.inf
    top = torch.where(chosen[:, :1], best[:, :1], 0.0)
    p = torch.where(chosen, torch.exp(best - top), 0.0)
    total = (p if renorm else torch.exp(x - top)).sum(dim=1, keepdim=True)
    gate = torch.where(chosen, p / total, 0.0)
    expert = torch.where(chosen, expert, -1)
    key = torch.where(chosen, expert, E).reshape(-1)
    order = torch.argsort(key, stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(T * k, device=dev)
    slot = torch.where(chosen.reshape(-1), slot, -1).reshape(T, k)
    offsets = torch.searchsorted(key[order].contiguous(), torch.arange(E + 1, device=dev))
    token = torch.where(torch.arange(T * k, device=dev) < offsets[E], order // k, -1)
    return dict(expert=expert.int(), gate=gate, offsets=offsets.int(), slot=slot.int(), token=token.int())


def prepare(case, seed):
    c, kind = case, case["kind"]
    B, L, E, k, D, F = c["B"], c["L"], c["E"], c["k"], c["D"], c["F"]
    T, M = B * L, B * L * k
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(1_000_003 * int(seed) + 17)
    randn = lambda *shape: torch.randn(shape, device=dev, generator=gen)  # noqa: E731
    bf16 = lambda t: t.to(torch.bfloat16)  # noqa: E731
    zeros = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    wide = torch.float32 if c["f32"] else torch.bfloat16
    st = dict(case=c, rows=None)
    if c["ragged"] < 1:
        lo = max(1, int(c["ragged"] * L))
        st["rows"] = torch.randint(lo, L + 1, (B,), device=dev, generator=gen).int()
    # experts differ in how often they are chosen, as trained routers' do
    logits = randn(T, E) + 0.5 * randn(E)
    if c["coarse"]:
        logits = bf16(logits).float()
    if c["masked"] > 0:
        logits[torch.rand((T, E), device=dev, generator=gen) < c["masked"]] = -math.inf
    r = _route(logits, st["rows"], B, L, k, c["renorm"])
    if kind.startswith("route"):
        st["logits"] = logits
        if kind == "route":
            st["out"] = dict(expert=zeros(T, k, dtype=torch.int32), gate=zeros(T, k), offsets=zeros(E + 1, dtype=torch.int32),
                             slot=zeros(T, k, dtype=torch.int32), token=zeros(M, dtype=torch.int32))
        else:
            st.update(expert=r["expert"], gate=r["gate"], dgate=randn(T, k), out=zeros(T, E))
        return st
    st.update(offsets=r["offsets"], token=r["token"], slot=r["slot"], gate=r["gate"])
    if kind.startswith("linear"):
        st["most"] = max(1, int((r["offsets"][1:] - r["offsets"][:-1]).max()))   # rows of the fullest expert
        if not c["gather"]:
            st["token"] = None
        if kind == "linear":
            st.update(X=bf16(randn(T if c["gather"] else M, D)), W=bf16(randn(E, F, D) / math.sqrt(D)), bias=0.02 * randn(E, F),
                      out=zeros(M, F, dtype=wide), pre=zeros(M, F, dtype=torch.bfloat16) if c["pre"] else None)
        elif kind == "linear_back_x":
            st.update(dY=bf16(randn(M, F)), W=bf16(randn(E, F, D) / math.sqrt(F)), pre=bf16(randn(M, D)) if c["gelu"] else None,
                      out=zeros(M, D, dtype=wide))
        else:
            st.update(dY=bf16(randn(M, F)), X=bf16(randn(T if c["gather"] else M, D)),
                      out=dict(dW=zeros(E, F, D, dtype=wide), dbias=zeros(E, F)))
        return st
    st.update(Y=bf16(randn(M, D)), res=bf16(randn(T, D)) if c["res"] else None, scale=1.25,
              gamma=1 + 0.1 * randn(D) if c["norm"] else None, beta=0.1 * randn(D) if c["norm"] else None)
    if kind == "combine":
        st["out"] = dict(sum=zeros(T, D, dtype=torch.bfloat16))
        if c["norm"]:
            st["out"]["out"] = zeros(T, D, dtype=torch.bfloat16)
    else:
        st.update(dsum=bf16(randn(T, D)), dout=bf16(randn(T, D)) if c["norm"] else None)
        st["out"] = dict(dY=zeros(M, D, dtype=torch.bfloat16), dgate=zeros(T, k))
        if c["res"]:
            st["out"]["dres"] = zeros(T, D, dtype=torch.bfloat16)
        if c["norm"]:
            st["out"].update(dgamma=zeros(D), dbeta=zeros(D))
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _workspace(sc, st):
    """The workspace a program keeps beside its weights."""
    if "ws" not in st:
        c = st["case"]
        st["ws"] = sc.new_expert_workspace(c["B"], c["L"], c["E"], c["k"], max(c["D"], c["F"], 8))
    return st["ws"]


def _run_own(st):
    import paper_2310_07109_gb300 as sc
    c, kind, ws = st["case"], st["case"]["kind"], _workspace(sc, st)
    B, L, rows, out = c["B"], c["L"], st["rows"], st["out"]
    if kind == "route":
        return sc.expert_route_forward(st["logits"], B=B, L=L, k=c["k"], rows=rows, renormalize=c["renorm"], out=out, workspace=ws)
    if kind == "route_back":
        return sc.expert_route_backward(st["logits"], st["expert"], st["gate"], st["dgate"], B=B, L=L, rows=rows,
                                        renormalize=c["renorm"], out=out)
    if kind == "linear":
        sc.expert_linear_forward(st["X"], st["W"], st["offsets"], token=st["token"], bias=st["bias"], gelu=c["gelu"],
                                 pre=st["pre"], out=out, workspace=ws)
        return (out, st["pre"]) if c["pre"] else out
    if kind == "linear_back_x":
        return sc.expert_linear_backward_input(st["dY"], st["W"], st["offsets"], pre=st["pre"], out=out, workspace=ws)
    if kind == "linear_back_w":
        return sc.expert_linear_backward_weight(st["dY"], st["X"], st["offsets"], token=st["token"], out=out, workspace=ws)
    block = dict(B=B, L=L, rows=rows, res=st["res"], res_scale=st["scale"], gamma=st["gamma"], eps=EPS, out=out)
    if kind == "combine":
        return sc.expert_combine_forward(st["Y"], st["slot"], st["gate"], beta=st["beta"], **block)
    return sc.expert_combine_backward(st["Y"], st["slot"], st["gate"], dout=st["dout"], dsum=st["dsum"], workspace=ws, **block)


def _gelu(x):
    return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))


def _gelu_slope(x):
    return 0.5 * (1 + torch.erf(x / math.sqrt(2))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _padded(t, index, inside):
    """Rows of t by expert, [E][most][...] in 32 bits, zero where an expert has no row."""
    return torch.where(inside[..., None], t[index].float(), 0.0)


def _run_plain(st):
    c, kind = st["case"], st["case"]["kind"]
    B, L, E, k = c["B"], c["L"], c["E"], c["k"]
    if kind == "route":
        return _route(st["logits"], st["rows"], B, L, k, c["renorm"])
    if kind == "route_back":
        x, gate = st["logits"], st["gate"]
        chosen = st["expert"] >= 0
        at = st["expert"].clamp(min=0).long()
        inner = (gate * st["dgate"]).sum(dim=1, keepdim=True)
        if c["renorm"]:
            return torch.zeros_like(x).scatter_add(1, at, torch.where(chosen, gate * (st["dgate"] - inner), 0.0))
        x = torch.where(x.isnan(), -math.inf, x)
        p = torch.exp(x - x.amax(dim=1, keepdim=True))
        p = p / p.sum(dim=1, keepdim=True)
        d = torch.zeros_like(x).scatter_add(1, at, torch.where(chosen, st["dgate"], 0.0))
        return torch.where(chosen[:, :1], p * (d - inner), 0.0)
    if kind.startswith("linear"):
        offsets = st["offsets"].long()
        index = offsets[:E, None] + torch.arange(st["most"], device=offsets.device)[None, :]
        inside = index < offsets[1:, None]
        M = B * L * k
        index = index.clamp(max=M - 1)
        slots = torch.arange(M, device=offsets.device)
        of = torch.searchsorted(offsets[1:].contiguous(), slots, right=True).clamp(max=E - 1)
        used = (slots < offsets[E])[:, None]
        at = (slots - offsets[of]).clamp(max=st["most"] - 1)
        rows_of_x = index if st["token"] is None else st["token"].long().clamp(min=0)[index]
        if kind == "linear_back_w":
            dy = _padded(st["dY"], index, inside)
            dw = torch.bmm(dy.transpose(1, 2), _padded(st["X"], rows_of_x, inside))
            return dict(dW=dw.to(st["out"]["dW"].dtype), dbias=dy.sum(dim=1))
        if kind == "linear":
            if M <= E:   # few slots: the chosen experts' weights alone
                x = st["X"][slots if st["token"] is None else st["token"].long().clamp(min=0)].float()
                y = (torch.bmm(st["W"][of].float(), x[:, :, None])[:, :, 0] + st["bias"][of])
            else:
                y = torch.bmm(_padded(st["X"], rows_of_x, inside), st["W"].float().transpose(1, 2)) + st["bias"][:, None, :]
                y = y[of, at]
            out = torch.where(used, _gelu(y) if c["gelu"] else y, 0.0).to(st["out"].dtype)
            return (out, torch.where(used, y, 0.0).to(torch.bfloat16)) if c["pre"] else out
        if M <= E:
            x = torch.bmm(st["dY"].float()[:, None, :], st["W"][of].float())[:, 0]
        else:
            x = torch.bmm(_padded(st["dY"], index, inside), st["W"].float())[of, at]
        if c["gelu"]:
            x = x * _gelu_slope(st["pre"].float())
        return torch.where(used, x, 0.0).to(st["out"].dtype)
    # combine and combine_back
    slot, D = st["slot"].long(), c["D"]
    here = torch.ones((B, L), dtype=torch.bool, device=slot.device)
    if st["rows"] is not None:
        here = torch.arange(L, device=slot.device)[None, :] < st["rows"][:, None]
    here = here.reshape(B * L, 1)
    y = torch.where((slot >= 0)[..., None], st["Y"][slot.clamp(min=0)].float(), 0.0)
    s = (st["gate"][..., None] * y).sum(dim=1)
    if c["res"]:
        s = s + st["scale"] * st["res"].float()
    if c["norm"]:
        centred = s - s.mean(dim=1, keepdim=True)
        inv = 1 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
        hat = centred * inv
    if kind == "combine":
        out = dict(sum=torch.where(here, s, 0.0).to(torch.bfloat16))
        if c["norm"]:
            out["out"] = torch.where(here, hat * st["gamma"] + st["beta"], 0.0).to(torch.bfloat16)
        return out
    ds = st["dsum"].float()
    out = {}
    if c["norm"]:
        do = torch.where(here, st["dout"].float(), 0.0)
        dh = do * st["gamma"]
        ds = ds + inv * (dh - dh.mean(dim=1, keepdim=True) - hat * (dh * hat).mean(dim=1, keepdim=True))
        out.update(dgamma=(do * hat).sum(dim=0), dbeta=do.sum(dim=0))
    ds = torch.where(here, ds, 0.0)
    out["dgate"] = (ds[:, None, :] * y).sum(dim=2)
    flat = torch.where(slot >= 0, slot, B * L * k).reshape(-1)
    dy = torch.zeros((B * L * k + 1, D), device=slot.device)
    dy[flat] = (st["gate"][..., None] * ds[:, None, :]).reshape(-1, D)
    out["dY"] = dy[:-1].to(torch.bfloat16)
    if c["res"]:
        out["dres"] = (st["scale"] * ds).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    """From the definitions, one expert (or one choice) at a time, in 64 bits; None where the values are whole."""
    st = prepare(case, seed)
    c, kind = case, case["kind"]
    B, L, E, k, D, F = c["B"], c["L"], c["E"], c["k"], c["D"], c["F"]
    T, M = B * L, B * L * k
    dev = torch.device("cuda", torch.cuda.current_device())
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=dev)  # noqa: E731
    lens = [L] * B if st["rows"] is None else st["rows"].tolist()
    used = torch.zeros(T, dtype=torch.bool, device=dev)
    for b, n in enumerate(lens):
        used[b * L: b * L + n] = True
    if kind.startswith("route"):
        x = torch.nan_to_num(st["logits"].double(), nan=-math.inf, posinf=math.inf, neginf=-math.inf)
        x[~used] = -math.inf
        left, picks, marks = x.clone(), [], []
        for _ in range(k):
            top = left.amax(dim=1)
            first = (left == top[:, None]).int().argmax(dim=1)     # the lowest expert at the maximum
            marks.append(top > -math.inf)
            picks.append(first)
            left = left.scatter(1, first[:, None], -math.inf)
        picks, marks = torch.stack(picks, 1), torch.stack(marks, 1)
        mask = torch.zeros((T, E), dtype=torch.bool, device=dev).scatter(1, picks, marks)
        for j in range(k):   # a later choice that is none must not clear an earlier one's mark
            mask |= torch.nn.functional.one_hot(picks[:, j], E).bool() & marks[:, j: j + 1]
        some = marks[:, 0]
        p = f64(T, E)
        sel = x.masked_fill(~mask, -math.inf) if c["renorm"] else x
        p[some] = torch.softmax(sel[some], dim=1)
        gate = torch.where(marks, p.gather(1, picks), 0.0)
        if kind == "route":
            return dict(expert=None, gate=gate, offsets=None, slot=None, token=None)
        dg = f64(T, E)
        for j in range(k):
            e = st["expert"][:, j].long()
            ok = torch.nonzero(e >= 0)[:, 0]
            dg[ok, e[ok]] = st["dgate"][ok, j].double()
        # d/dl of sum_e dg_e p_e: p is a softmax (over the chosen, or over all)
        return p * (dg - (p * dg).sum(dim=1, keepdim=True))
    if kind.startswith("linear"):
        off = st["offsets"].tolist()
        token = None if st["token"] is None else st["token"].long()
        rows = lambda t, a, b: t[a:b].double() if token is None else t[token[a:b]].double()  # noqa: E731
        norm = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device=dev), 1.0)
        if kind == "linear_back_w":
            dW, db = f64(E, F, D), f64(E, F)
            for e in range(E):
                a, b = off[e], off[e + 1]
                dy = st["dY"][a:b].double()
                dW[e], db[e] = dy.T @ rows(st["X"], a, b), dy.sum(dim=0)
            return dict(dW=dW, dbias=db)
        out = f64(M, F if kind == "linear" else D)
        pre = f64(*out.shape) if c["pre"] else None
        for e in range(E):
            a, b = off[e], off[e + 1]
            if kind == "linear":
                y = rows(st["X"], a, b) @ st["W"][e].double().T + st["bias"][e].double()
                if c["pre"]:
                    pre[a:b] = y
                out[a:b] = y * norm.cdf(y) if c["gelu"] else y
            else:
                y = st["dY"][a:b].double() @ st["W"][e].double()
                if c["gelu"]:
                    z = st["pre"][a:b].double()
                    y = y * (norm.cdf(z) + z * torch.exp(norm.log_prob(z)))
                out[a:b] = y
        return (out, pre) if c["pre"] else out
    Y = st["Y"].double()
    s = f64(T, D) if st["res"] is None else st["scale"] * st["res"].double()
    s[~used] = 0
    picked = []
    for j in range(k):
        at = st["slot"][:, j].long()
        row = Y[at.clamp(min=0)] * (at >= 0)[:, None]
        picked.append(row)
        s = s + st["gate"][:, j: j + 1].double() * row
    if kind == "combine":
        out = dict(sum=s)
        if c["norm"]:
            out["out"] = torch.nn.functional.layer_norm(s, (D,), st["gamma"].double(), st["beta"].double(), EPS) * used[:, None]
        return out
    out, ds = {}, st["dsum"].double() * used[:, None]
    if c["norm"]:
        with torch.enable_grad():
            x = s.clone().requires_grad_(True)
            gamma, beta = st["gamma"].double().requires_grad_(True), st["beta"].double().requires_grad_(True)
            y = torch.nn.functional.layer_norm(x, (D,), gamma, beta, EPS)
            dx, out["dgamma"], out["dbeta"] = torch.autograd.grad(y, (x, gamma, beta), st["dout"].double() * used[:, None])
        ds = ds + dx
    out["dgate"] = torch.stack([(ds * row).sum(dim=1) for row in picked], dim=1)
    out["dY"] = f64(M, D)
    for j in range(k):
        at = st["slot"][:, j].long()
        ok = torch.nonzero(at >= 0)[:, 0]
        out["dY"][at[ok]] = st["gate"][ok, j: j + 1].double() * ds[ok]
    if st["res"] is not None:
        out["dres"] = st["scale"] * ds
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    """Inputs and outputs once each, at the expected number of rows in use; the weights of at most as many experts as
    there are slots."""
    c, kind = case, case["kind"]
    E, k, D, F = c["E"], c["k"], c["D"], c["F"]
    T = c["B"] * c["L"] * (1 + c["ragged"]) / 2
    M, busy = T * k, min(E, c["B"] * c["L"] * k)
    wide = 4 if c["f32"] else 2
    if kind == "route":
        return {"bytes": T * (4 * E + 12 * k) + 4 * M + 4 * E, "flops": 4 * T * E}
    if kind == "route_back":
        return {"bytes": T * (8 * E + 12 * k), "flops": 4 * T * E}
    if kind == "linear":
        x = min(T, M) if c["gather"] else M
        return {"bytes": 2 * x * D + busy * (2 * D * F + 4 * F) + M * F * (wide + (2 if c["pre"] else 0)) + 4 * M * c["gather"],
                "flops": 2 * M * D * F}
    if kind == "linear_back_x":
        return {"bytes": 2 * M * F + busy * 2 * D * F + M * D * (wide + (2 if c["gelu"] else 0)), "flops": 2 * M * D * F}
    if kind == "linear_back_w":
        x = min(T, M) if c["gather"] else M
        return {"bytes": 2 * x * D + 2 * M * F + E * F * (D * wide + 4) + 4 * M * c["gather"], "flops": 2 * M * D * F + M * F}
    if kind == "combine":
        return {"bytes": M * (2 * D + 8) + T * D * 2 * (c["res"] + 1 + c["norm"]), "flops": T * D * (2 * k + 2 + 8 * c["norm"])}
    return {"bytes": M * (4 * D + 12) + T * D * 2 * (2 * c["res"] + 1 + c["norm"]) + 8 * D * c["norm"],
            "flops": T * D * (6 * k + 2 + 16 * c["norm"])}
