"""Plain implementations that the cache tests compare with, on the CPU: the 4-bit
values element by element, a page byte by byte, and attention over positions in
64 bits."""
import math

import torch

from tests.attnref import U32, UBF

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def quantise(x):
    """Codes [..., d] and scale bytes [..., d / 32] of float64 rows: the nearest of the
    sixteen values by distance, between two as near the one with an even code."""
    y = x.unflatten(-1, (-1, 32))
    m = y.abs().amax(-1)
    bad = ~torch.isfinite(y).all(-1)
    e = torch.full_like(m, -125.0)
    for k in range(-125, 127):              # the least e with m <= 7 2^e
        e = torch.where((m > 7.0 * 2.0 ** k) & ~bad, torch.full_like(e, k + 1.0), e)
    z = torch.where(bad[..., None], torch.zeros_like(y), y) / torch.exp2(e)[..., None]
    gap = (z.abs()[..., None] - GRID).abs()
    odd = torch.arange(8) % 2
    best = (gap + 1e-12 * odd * (gap == gap.amin(-1, keepdim=True))).argmin(-1)
    code = best + 8 * torch.signbit(z)
    return code.flatten(-2), torch.where(bad, torch.full_like(e, 255.0), e + 127).long()


def values(code, exp):
    """What codes and scale bytes stand for."""
    v = GRID[code & 7] * torch.where(code >= 8, -1.0, 1.0)
    s = torch.where(exp == 255, torch.full_like(exp, 0, dtype=torch.float64) + math.nan,
                    torch.exp2(exp.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def put(page, j, kc, ke, vc, ve):
    """Token j's codes [d] and scale bytes [d / 32] into a page of bytes (uint8 [68 d])."""
    d = kc.numel()
    nb, a, g4, i, r = d // 32, j // 16, j // 4 % 4, j % 4, j % 16
    for ch in range(0, d, 2):
        blk, g, byte = ch // 32, ch % 32 // 8, ch % 8 // 2
        page[((j * 4 + g) * nb + blk) * 4 + byte] = int(kc[ch]) | int(kc[ch + 1]) << 4
        page[34 * d + (((blk * 16 + ch % 32 // 2) * 4 + g4) * 4 + a) * 4 + i] = int(vc[ch]) | int(vc[ch + 1]) << 4
    for blk in range(nb):
        page[32 * d + (blk * 16 + r) * 4 + a] = int(ke[blk])
        page[66 * d + ((blk * 4 + g4) * 4 + a) * 4 + i] = int(ve[blk])


def held(start, n, P):
    """Positions that a sequence holds once n tokens from `start` on are in."""
    end = start + n
    return range(max(0, ((end - 1) // 64 - P + 1) * 64), end) if end > 0 else range(0)


def attend(q, kv, starts, lengths, P, left, scale, missing=()):
    """out, lse and their largest errors (P in terms of 2^-16 for bf16, 0 for fp32): q
    [B, H, T, d] float64; kv[b]: (k, v) [HK, n, d] at every position; missing: pairs (b,
    page) that no page stands for."""
    B, H, T, d = q.shape
    out, lse = torch.zeros_like(q), torch.full(q.shape[:3], -math.inf, dtype=torch.float64)
    parts = []
    for b in range(B):
        k, v = (x.repeat_interleave(H // x.shape[0], 0) for x in kv[b])
        hold = held(starts[b], lengths[b], P)
        for t in range(lengths[b]):
            p = starts[b] + t
            j = [x for x in hold if (left < 0 or x >= p - left) and x <= p and (b, x // 64) not in missing]
            if p < 0 or not j:
                continue
            s = scale * (k[:, j] @ q[b, :, t, :, None])[..., 0]
            lse[b, :, t] = torch.logsumexp(s, -1)
            w = torch.exp(s - lse[b, :, t, None])
            out[b, :, t] = (w[:, None] @ v[:, j])[:, 0]
            big = scale * (k[:, j].abs() @ q[b, :, t, :, None].abs())[..., 0]
            e = U32 * (d + 4) * big + 4 * U32 * (lse[b, :, t, None].abs() + big.amax(-1, keepdim=True))
            e = e + (w * e).sum(-1, keepdim=True) + U32 * (len(j) + 16) + 2 * U32 * lse[b, :, t, None].abs()
            parts.append((b, t, w, e, v[:, j].abs(), len(j)))

    def bounds(bf):
        eo, el = torch.zeros_like(out), torch.zeros_like(out[..., 0])
        for b, t, w, e, av, n in parts:
            op = 2.0 ** -16 if bf else 2.0 ** -23
            eo[b, :, t] = ((w * (e + op + U32 * (n + 16)))[:, None] @ av)[:, 0] + \
                ((UBF if bf else 0.0) + 2 * U32) * out[b, :, t].abs()
            el[b, :, t] = (w * e).sum(-1) + 4 * U32 * lse[b, :, t].abs()
        return 1.01 * eo + 1e-30, 1.01 * el + 1e-30
    return out, lse, bounds
