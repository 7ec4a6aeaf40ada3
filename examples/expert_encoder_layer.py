"""An encoder layer with a mixture-of-experts feed-forward block, forward and one training step.

The layer's sparse attention drops tokens; the block runs on the ones it keeps, whose number is known
on the device alone.  A router sends each kept token to k of E experts; every product below works on
ragged groups of rows (``offsets``), and no size comes back to the host:

    Q, K, V        = X W_qkv^T + b_qkv                           linear_forward
    O, kept tokens = sparse attention with token pruning         layer_forward
    H  = LN(X[kept] + O[kept] W_o^T + b_o)                       linear_forward, layer_norm_forward
    l  = H W_r^T                                                 expert_linear_forward, one group
    g, slots       = the k best experts of each token            expert_route_forward
    F  = GELU(H[token] W_1e^T + b_1e)                            expert_linear_forward
    Z  = F W_2e^T + b_2e                                         expert_linear_forward
    Y  = LN(H + sum_j g_j Z[slot_j])                             expert_combine_forward

Run on a GPU:  python examples/expert_encoder_layer.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2310_07109_gb300 as sc

EPS = 1e-5


class ExpertFeedForward:
    """Router, experts and the block's end; fp32 parameters, bf16 copies for the products."""

    def __init__(self, D, F, E, k, *, device="cuda", seed=0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, device=device, generator=g)  # noqa: E731
        self.D, self.F, self.E, self.k = D, F, E, k
        self.params = {"W_r": randn(1, E, D) / math.sqrt(D),
                       "W_1": randn(E, F, D) / math.sqrt(D), "b_1": torch.zeros(E, F, device=device),
                       "W_2": randn(E, D, F) / math.sqrt(F), "b_2": torch.zeros(E, D, device=device),
                       "gamma": torch.ones(D, device=device), "beta": torch.zeros(D, device=device)}
        self.cast()

    def cast(self):
        self.half = {n: self.params[n].to(torch.bfloat16) for n in ("W_r", "W_1", "W_2")}

    def forward(self, H, B, L, rows, workspace=None):
        """H bf16 [B*L, D], rows int32 [B] in use.  Returns Y and what the backward pass needs."""
        p, w, ws = self.params, self.half, workspace
        if ws is None:
            ws = sc.new_expert_workspace(B, L, self.E, self.k, max(self.D, self.F), H.device)
        every = torch.arange(0, 2 * B * L, B * L, dtype=torch.int32, device=H.device)   # all rows, no copy from the host
        logits = sc.expert_linear_forward(H, w["W_r"], every, out_f32=True, workspace=ws)
        r = sc.expert_route_forward(logits, k=self.k, B=B, L=L, rows=rows, workspace=ws)
        pre = torch.empty(B * L * self.k, self.F, dtype=torch.bfloat16, device=H.device)
        F = sc.expert_linear_forward(H, w["W_1"], r["offsets"], token=r["token"], bias=p["b_1"], gelu=True,
                                     pre=pre, workspace=ws)
        Z = sc.expert_linear_forward(F, w["W_2"], r["offsets"], bias=p["b_2"], workspace=ws)
        out = {"out": torch.zeros(B * L, self.D, dtype=torch.bfloat16, device=H.device)}
        sc.expert_combine_forward(Z, r["slot"], r["gate"], B=B, L=L, rows=rows, res=H, gamma=p["gamma"],
                                  beta=p["beta"], eps=EPS, out=out)
        return out["out"], dict(H=H, B=B, L=L, rows=rows, every=every, logits=logits, route=r, pre=pre, F=F, Z=Z, ws=ws)

    def backward(self, dY, c):
        """dY bf16 [B*L, D], the gradient of Y.  Returns (gradients of the parameters, of H)."""
        p, w, r, ws = self.params, self.half, c["route"], c["ws"]
        shape = dict(B=c["B"], L=c["L"], rows=c["rows"])
        end = sc.expert_combine_backward(c["Z"], r["slot"], r["gate"], res=c["H"], gamma=p["gamma"], eps=EPS,
                                         dout=dY, workspace=ws, **shape)
        two = sc.expert_linear_backward_weight(end["dY"], c["F"], r["offsets"], workspace=ws)
        dpre = sc.expert_linear_backward_input(end["dY"], w["W_2"], r["offsets"], pre=c["pre"], workspace=ws)
        one = sc.expert_linear_backward_weight(dpre, c["H"], r["offsets"], token=r["token"], workspace=ws)
        dslots = sc.expert_linear_backward_input(dpre, w["W_1"], r["offsets"], workspace=ws)
        dlogits = sc.expert_route_backward(c["logits"], r["expert"], r["gate"], end["dgate"], **shape).to(torch.bfloat16)
        # rows that are not in use hold anything: the router's product over all rows takes zeros there
        live = (torch.arange(c["L"], device=dY.device)[None, :] < c["rows"][:, None]).reshape(-1, 1)
        router = sc.expert_linear_backward_weight(dlogits, torch.where(live, c["H"], 0), c["every"], bias=False, workspace=ws)
        dH = sc.expert_linear_backward_input(dlogits, w["W_r"], c["every"], workspace=ws)
        # a token's gradient: from the residual, from its slots, from the router
        dH = sc.expert_combine_forward(dslots, r["slot"], None, res=torch.where(live, end["dres"] + dH, 0), **shape)["sum"]
        return {"W_r": router["dW"], "W_1": one["dW"], "b_1": one["dbias"], "W_2": two["dW"], "b_2": two["dbias"],
                "gamma": end["dgamma"], "beta": end["dbeta"]}, dH

    def step(self, grads, rate):
        for name, grad in grads.items():
            self.params[name] -= rate * grad
        self.cast()


def attention_half(X, weights, w, alpha):
    """The layer up to the feed-forward block: (H [B*L, D] of the kept tokens, their number per sequence)."""
    B, L, D = X.shape
    heads = D // 64
    dev = X.device
    length = torch.full((B,), L, dtype=torch.int32, device=dev)
    pos = torch.arange(L, dtype=torch.int32, device=dev).repeat(B, 1)
    qkv = sc.linear_forward(X, weights["W_qkv"], B=B, L=L, bias=weights["b_qkv"])
    q, k, v = (t.contiguous().view(B, L, heads, 64) for t in qkv.split(D, dim=1))
    O, _, kept, rows = sc.layer_forward(q, k, v, length, pos, w, [0], alpha)
    # before the first pruning a token's position is its row
    S = sc.linear_forward(O.view(B * L, D), weights["W_o"], B=B, L=L, rows=rows, gidx=kept, bias=weights["b_o"],
                          res=X, res_gathered=True, out_f32=True)
    H = sc.layer_norm_forward(S, weights["ln_gamma"], weights["ln_beta"], B=B, L=L, rows=rows)
    return H, rows


def attention_weights(D, device="cuda", seed=1):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    mat = lambda o, i: (torch.randn(o, i, device=device, generator=g) / math.sqrt(i)).to(torch.bfloat16)  # noqa: E731
    return {"W_qkv": mat(3 * D, D), "b_qkv": torch.zeros(3 * D, device=device), "W_o": mat(D, D),
            "b_o": torch.zeros(D, device=device), "ln_gamma": torch.ones(D, device=device),
            "ln_beta": torch.zeros(D, device=device)}


def main(B=4, L=512, D=768, F=1536, E=8, k=2, steps=8, quiet=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    X = torch.randn(B, L, D, device="cuda", generator=g).to(torch.bfloat16)
    target = torch.randn(B * L, D, device="cuda", generator=g)
    H, rows = attention_half(X, attention_weights(D), 64, 0.7)
    live = (torch.arange(L, device="cuda")[None, :] < rows[:, None]).reshape(-1, 1)
    block = ExpertFeedForward(D, F, E, k)
    losses = []
    for _ in range(steps):
        Y, saved = block.forward(H, B, L, rows)
        diff = torch.where(live, Y.float() - target, 0.0)
        losses.append(diff.square().sum() / (2 * live.sum()))
        grads, _ = block.backward((diff / live.sum()).to(torch.bfloat16), saved)
        block.step(grads, 0.2)
    losses = [float(x) for x in losses]
    if not quiet:
        print("kept %s of %d tokens a sequence; slots of the experts %s" % (
            rows.tolist(), L, (saved["route"]["offsets"][1:] - saved["route"]["offsets"][:-1]).tolist()))
        print("loss " + " ".join("%.4f" % x for x in losses))
    status = sc.workspace_status(saved["ws"])
    assert status == sc.SC_OK, sc.status_string(status)
    return losses


if __name__ == "__main__":
    main()
