"""The rotation of heads and the pruned key-value cache from their definitions, in 64 bits: plain
loops over sequences, lists and heads, sharing nothing with the kernels."""
import math

import torch


def eps_of(dtype):
    """Half a step: what one rounding to ``dtype`` may change of a value."""
    return torch.finfo(dtype).eps / 2


def head(x, gamma, eps, pos, freq, inter, m):
    """x [..., d] of heads whose tokens are at pos [..., 1]; freq [rot / 2] or None."""
    y = x.double()
    if gamma is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gamma.double()
    if freq is None:
        return y
    n = freq.numel()
    a = pos.double() * freq
    cos, sin = m * torch.cos(a), m * torch.sin(a)
    first = torch.arange(0, 2 * n, 2) if inter else torch.arange(n)
    second = first + 1 if inter else first + n
    out = y.clone()
    out[..., first] = y[..., first] * cos - y[..., second] * sin
    out[..., second] = y[..., second] * cos + y[..., first] * sin
    return out


def heads(x, H, d, gamma, eps, pos, freq, inter, m):
    """x [T, H d], pos [T]: [T, H d] in 64 bits."""
    T = x.shape[0]
    return head(x.reshape(T, H, d), gamma, eps, pos[:, None, None], freq, inter, m).reshape(T, H * d)


def pair_size(y, freq, inter):
    """For each feature the length of its pair (itself where it is not rotated); y [T, H, d]."""
    out = y.abs()
    if freq is None:
        return out
    n = freq.numel()
    first = torch.arange(0, 2 * n, 2) if inter else torch.arange(n)
    second = first + 1 if inter else first + n
    size = torch.hypot(y[..., first], y[..., second])
    out[..., first] = size
    out[..., second] = size
    return out


def attend(cache, Q, T, rows, scale, decay):
    """(O, acc, slack of O, slack of acc): from the cache's tensors as they are; rows a list.  The slack is how far
    scores of 32-bit sums, weights and their sums may be off before the one rounding of O: a sum of d products is within
    (d + 16) 2^-23 of their magnitudes, a weight within twice its score's error, 2^-20 for the
    exponentials and the logarithm, and half a step of the 16-bit type where it meets V."""
    K, V, acc, pos = cache["K"].double(), cache["V"].double(), cache["acc"].double(), cache["pos"]
    B, Hk, C, d = K.shape
    G = acc.shape[1]
    H = Q.shape[1] // d
    u = eps_of(Q.dtype)
    O = torch.zeros(B * T, H, d, dtype=torch.float64, device=K.device)  # noqa: E741
    slack = torch.zeros_like(O)
    new, acc_slack = acc.clone(), torch.zeros_like(acc)
    q = Q.double().reshape(B * T, H, d)
    for b in range(B):
        first = int(cache["seen"][b]) - rows[b]
        for g in range(G):
            n = min(max(int(cache["len"][b, g]), 0), C)
            if rows[b] > 0:
                new[b, g, :n] *= decay
                acc_slack[b, g, :n] = new[b, g, :n].abs() * 2.0 ** -22
            for r in range(rows[b]):
                at = pos[b, g, :n]
                see = torch.nonzero((at >= 0) & (at <= first + r))[:, 0]
                if len(see) == 0:
                    continue
                for h in range(g * H // G, (g + 1) * H // G):
                    k, v, x = K[b, h * Hk // H, see], V[b, h * Hk // H, see], q[b * T + r, h]
                    s = scale * (k @ x)
                    off = 2 * float((k.abs() @ x.abs()).max()) * abs(scale) * (d + 16) * 2.0 ** -23 + 2.0 ** -20
                    off += float(s.abs().max()) * 2.0 ** -22
                    p = torch.softmax(s, 0)
                    O[b * T + r, h] = p @ v
                    slack[b * T + r, h] = (p @ v.abs()) * (off + u * 1.01 + len(see) * 2.0 ** -23)
                    new[b, g, see] += p / (H // G)
                    acc_slack[b, g, see] += p / (H // G) * (off + (rows[b] * H + 16) * 2.0 ** -23)
    return O.reshape(B * T, H * d), new, slack.reshape(B * T, H * d), acc_slack


def survivors(acc, pos, n, seen, budget, slack, sinks, recent):
    """(source of each of the first slots after eviction): lists of plain numbers."""
    if n <= budget + slack:
        return list(range(n))

    def rank(i):
        if pos[i] < 0 or (math.isnan(acc[i]) and not (pos[i] < sinks or pos[i] >= seen - recent)):
            return (2, 0.0, i)
        if pos[i] < sinks or pos[i] >= seen - recent:
            return (0, 0.0, i)
        return (1, -acc[i], i)

    kept = sorted(sorted(range(n), key=rank)[:budget])
    stay, fill = {i for i in kept if i < budget}, [i for i in kept if i >= budget]
    return [i if i in stay else fill.pop(0) for i in range(budget)]


def evict(cache, budget, slack, sinks, recent):
    """(K, V, acc, pos, len) afterwards; slots from len on as they were."""
    K, V, acc, pos, length = (cache[n].clone() for n in ("K", "V", "acc", "pos", "len"))
    B, Hk, C, _ = K.shape
    G = acc.shape[1]
    for b in range(B):
        for g in range(G):
            n = min(max(int(length[b, g]), 0), C)
            src = survivors(acc[b, g, :n].tolist(), pos[b, g, :n].tolist(), n, int(cache["seen"][b]), budget, slack, sinks, recent)
            at = torch.tensor(src, dtype=torch.long, device=K.device)
            own = slice(g * Hk // G, (g + 1) * Hk // G)
            for t in (K, V):
                t[b, own, :len(src)] = t[b, own][:, at]
            for t in (acc, pos):
                t[b, g, :len(src)] = t[b, g, at]
            length[b, g] = len(src)
    return K, V, acc, pos, length
