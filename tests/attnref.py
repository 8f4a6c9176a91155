"""Plain 64-bit attention that the tests compare with, on the CPU: the softmax
over the keys a query sees, its gradients written out, and how far a result in
fewer bits may be from them, element by element."""
import math

import torch

U32, UBF = 2.0 ** -24, 2.0 ** -8      # half a step, relative to the value


def seen(B, T, S, left, right, lengths):
    """[B, T, S]: whether query t sees key j."""
    p = torch.arange(T)[:, None] + (S - T)
    j = torch.arange(S)[None, :]
    m = torch.ones(T, S, dtype=torch.bool)
    if left >= 0:
        m &= j >= p - left
    if right >= 0:
        m &= j <= p + right
    end = (torch.full((B,), T) if lengths is None else lengths.clamp(0, T)).view(B, 1, 1) + (S - T)
    return m & (j < end) & (p < end)


def heads(x, H):
    return x.repeat_interleave(H // x.shape[1], 1)


def groups(x, HK):
    return x.unflatten(1, (HK, -1)).sum(2)


def clean(x, m):
    """Rows that nothing reads, as zeros."""
    return torch.where(m[:, None, :, None], x, torch.zeros((), dtype=x.dtype))


def attention(x, scale, left, right, lengths):
    """out, lse, P of x = dict(q, k, v) in float64 (tokens that are not live may hold anything)."""
    B, H, T, _ = x["q"].shape
    S = x["k"].shape[2]
    m = seen(B, T, S, left, right, lengths)
    live = torch.arange(T) < (torch.full((B,), T) if lengths is None else lengths.clamp(0, T))[:, None]
    keys = torch.arange(S) < live.sum(-1, keepdim=True) + (S - T)
    q, k, v = clean(x["q"], live), heads(clean(x["k"], keys), H), heads(clean(x["v"], keys), H)
    s = (scale * (q @ k.transpose(-1, -2))).masked_fill(~m[:, None], -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None])
    return p @ v, lse, dict(p=p, q=q, k=k, v=v, m=m, live=live)


def gradients(x, scale, left, right, lengths, d_out, d_lse=None):
    """out, lse, {q, k, v: gradient}, and the parts that the bounds are made of."""
    out, lse, a = attention(x, scale, left, right, lengths)
    HK = x["k"].shape[1]
    g = clean(d_out, a["live"])
    D = (g * out).sum(-1)
    if d_lse is not None:
        D = D - torch.where(lse == -math.inf, torch.zeros_like(lse), d_lse)
    u = g @ a["v"].transpose(-1, -2)
    ds = a["p"] * (u - D[..., None])
    a.update(g=g, ds=ds, u=u, D=D)
    return out, lse, dict(q=scale * (ds @ a["k"]), k=scale * groups(ds.transpose(-1, -2) @ a["q"], HK),
                          v=groups(a["p"].transpose(-1, -2) @ g, HK)), a


def bounds(a, out, lse, scale, HK, bf):
    """Largest errors of out, lse and the gradients.

    Sums of n products in fp32 lose at most n 2^-24 of the sum of their magnitudes.
    A probability is e^(score - lse): its error is P times that of the exponent (the
    score's, the lse's, two roundings of the scaled difference) and a few 2^-24, and all
    of it where it is no normal number of fp32.  With bf16 a P or dS is off by another 2^-8 as an operand, and what is written by 2^-8."""
    ub = UBF if bf else 0.0
    d, n, nq = a["q"].shape[-1], a["k"].shape[2], a["q"].shape[2] * (a["q"].shape[1] // HK)
    big = scale * (a["q"].abs() @ a["k"].abs().transpose(-1, -2))
    lsz = torch.where(lse == -math.inf, torch.zeros_like(lse), lse).abs()
    e_s = U32 * (d + 4) * big + 4 * U32 * (lsz[..., None] + big.amax(-1, keepdim=True))
    e_lse = (a["p"] * e_s).sum(-1) + U32 * (n + 8) + 2 * U32 * lsz
    tiny = 2.0 ** -125          # (what is below 2^-126 is zero, before and after a rounding)
    e_p = a["p"] * (e_s + e_lse[..., None] + 8 * U32) + tiny
    av = a["v"].abs()
    e_out = (ub * a["p"] + e_p + U32 * (n + 8) * a["p"]) @ av + (ub + 2 * U32) * out.abs()
    res = dict(out=1.01 * e_out + 1e-30, lse=e_lse)
    if "ds" not in a:
        return res
    ga = a["g"].abs()
    e_D = (ga * e_out).sum(-1) + U32 * (d + 4) * (ga * out.abs()).sum(-1) + 2 * U32 * a["D"].abs()
    e_u = U32 * (d + 2) * (ga @ av.transpose(-1, -2))
    e_ds = e_p * (a["u"] - a["D"][..., None]).abs() + (a["p"] + e_p) * (e_D[..., None] + e_u) + 4 * U32 * a["ds"].abs() + tiny
    ads, ap, aq, ak = a["ds"].abs(), a["p"], a["q"].abs(), a["k"].abs()
    t = lambda m: m.transpose(-1, -2)
    w_q = scale * ((ub + U32 * (n + 8)) * ads + (1 + ub) * e_ds) @ ak
    w_k = scale * groups(t((ub + U32 * (nq + 8)) * ads + (1 + ub) * e_ds) @ aq, HK)
    w_v = groups(t((ub + U32 * (nq + 8)) * ap + (1 + ub) * e_p) @ ga, HK)
    return dict(res, q=w_q, k=w_k, v=w_v, own=ub + 2 * U32)
