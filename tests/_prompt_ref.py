"""Packed prompts' attention and the weight it leaves, and log probabilities, in 64 bits
from their definitions; and how far binary32 with the roundings that the header names may
be from them."""
import math

import torch


def spans(starts):
    return list(zip(starts, starts[1:]))


def attend(q, k, v, starts, scale):
    """out, lse and their bounds, all float64, NaN outside the sequences."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=q.device)  # noqa: E731
    out, lse, far_out, far_lse = nan(T, Hq, D), nan(T, Hq), nan(T, Hq, D), nan(T, Hq)
    for a, z in spans(starts):
        n = z - a
        if n <= 0:
            continue
        unseen = torch.ones((n, n), dtype=torch.bool, device=q.device).triu(1)
        for head in range(Hq):
            kk, vv, qq = k[a:z, head // G], v[a:z, head // G], q[a:z, head]
            s = (scale * (qq @ kk.T)).masked_fill(unseen, -math.inf)
            m = s.amax(1, keepdim=True)
            p = torch.exp(s - m)
            total = p.sum(1, keepdim=True)
            p = p / total
            lse[a:z, head] = (m + total.log())[:, 0]
            out[a:z, head] = p @ vv
            # a score: D products and sums, scaled; its exponential: that, its argument's
            # rounding, and the function's; sums of n terms
            size = abs(scale) * (qq.abs() @ kk.abs().T).masked_fill(unseen, 0.0).amax(1, keepdim=True)
            e = size * (D + 4) * 2.0 ** -23 + (m.abs() + 40) * 2.0 ** -23 + (n + 8) * 2.0 ** -24
            # weights to bf16 and out to bf16 are half a step each, 2^-8
            far_out[a:z, head] = (2.0 ** -8 + 2 * e) * (p @ vv.abs()) + 2.0 ** -8 * out[a:z, head].abs()
            far_lse[a:z, head] = (e + lse[a:z, head].abs()[:, None] * 2.0 ** -23)[:, 0]
    return out, lse, far_out * (1 + 2.0 ** -6), far_lse


def weigh(q, k, lse, starts, last, scale):
    """weight (H, T) and its bound, NaN outside the sequences."""
    T, Hq, D = q.shape
    H = k.shape[1]
    q, k, lse = q.double(), k.double(), lse.double()
    weight = torch.full((H, T), math.nan, dtype=torch.float64, device=q.device)
    far = weight.clone()
    for a, z in spans(starts):
        if z <= a:
            continue
        weight[:, a:z], far[:, a:z] = 0.0, 0.0
        first = max(a, z - last)
        for head in range(Hq):
            h = head // (Hq // H)
            qq, kk = q[first:z, head], k[a:z, h]
            seen = torch.ones((z - first, z - a), dtype=torch.bool, device=q.device).tril(first - a)
            l = lse[first:z, head, None]
            seen &= l != -math.inf
            s = scale * (qq @ kk.T)
            p = torch.where(seen, torch.exp(s - l), 0.0)
            e = abs(scale) * (qq.abs() @ kk.abs().T) * (D + 4) * 2.0 ** -23 + (s.abs() + l.abs() + 4) * 2.0 ** -22
            weight[h, a:z] += p.sum(0)
            far[h, a:z] += torch.where(seen, p * e, 0.0).sum(0)
        far[:, a:z] += weight[:, a:z] * ((z - first) * (Hq // H) + 8) * 2.0 ** -24
    return weight, far + 2.0 ** -126


def logprobs(x, tokens, top):
    """One request's rows x (N, V), tokens (N, M): log p of all, entropy, top tokens, and bounds of the
    log probabilities (N, 1) past 2^-23 of their size, and of the entropy (N,)."""
    V = x.shape[1]
    y = torch.log_softmax(x.double(), 1)
    p = y.exp()
    entropy = -torch.where(p > 0, p * y, 0.0).sum(1)
    # sums: V terms in lanes, steps and waves, at most V / 2^11 + 40 additions one after the other
    adds = (V / 2 ** 11 + 40) * 2.0 ** -24
    far = adds + (4 + entropy) * 2.0 ** -22
    order = torch.sort(torch.where(x.isnan(), -math.inf, x.double()), dim=1, descending=True, stable=True)
    ids = torch.where(order.values > -math.inf, order.indices, -1)[:, :top]
    if top > V:
        ids = torch.cat([ids, torch.full((x.shape[0], top - V), -1, device=x.device)], 1)
    return y, entropy, ids, far, far * (1 + entropy)
