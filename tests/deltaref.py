"""Plain 64-bit implementations that the delta rule and query/key tests compare
with: the recurrence token by token and the preparation row by row, on the CPU,
with gradients by torch.autograd."""
import torch


def repeat(x, H):
    return x.repeat_interleave(H // x.shape[1], 1)


def delta(q, k, v, eta, log_gamma, w, scale, lengths=None):
    """(out, w) of the gated delta rule; every argument float64."""
    B, H, T, _ = v.shape
    q, k = repeat(q, H), repeat(k, H)
    outs = []
    for t in range(T):
        live = torch.ones(B, 1, 1, 1, dtype=torch.bool) if lengths is None else \
            (t < lengths).view(B, 1, 1, 1)
        zero = torch.zeros((), dtype=torch.float64)
        kt = torch.where(live[..., 0], k[:, :, t], zero)
        qt = torch.where(live[..., 0], q[:, :, t], zero)
        vt = torch.where(live[..., 0], v[:, :, t], zero)
        et = torch.where(live[..., 0, 0], eta[:, :, t], zero)
        if log_gamma is not None:
            w = w * torch.where(live[..., 0, 0], log_gamma[:, :, t], zero).exp()[..., None, None]
        e = vt - (w @ kt[..., None])[..., 0]
        w = w + (et[..., None] * e)[..., None] * kt[..., None, :]
        outs.append(scale * (w @ qt[..., None])[..., 0])
    return torch.stack(outs, 2), w


def delta_grads(x, scale, d_out, d_w_out, lengths=None):
    """out, w_out and the gradients of x = dict(q, k, v, eta, log_gamma, w_in) (float64)."""
    leaves = {n: t.detach().clone().requires_grad_(True) for n, t in x.items() if t is not None}
    w = leaves.get("w_in")
    if w is None:
        B, H, _, dv = x["v"].shape
        w = torch.zeros(B, H, dv, x["q"].shape[-1], dtype=torch.float64)
    out, w_out = delta(leaves["q"], leaves["k"], leaves["v"], leaves["eta"], leaves.get("log_gamma"),
                       w, scale, lengths)
    loss = (out * d_out).sum() + (0 if d_w_out is None else (w_out * d_w_out).sum())
    grads = torch.autograd.grad(loss, list(leaves.values()))
    return out.detach(), w_out.detach(), dict(zip(leaves, grads))


def qk_row(x, inv_freq, positions, rot, silu, unit, interleaved, eps, m):
    """One tensor [B, H, T, d] of the query/key preparation, float64."""
    y = x * torch.sigmoid(x) if silu else x
    if unit:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) + eps)
    if not rot:
        return y
    a = positions.double()[:, None, :, None] * inv_freq.double()
    co, si = m * torch.cos(a), m * torch.sin(a)
    half = rot // 2
    if interleaved:
        p, q = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        p, q = y[..., :half], y[..., half:rot]
    zp, zq = p * co - q * si, q * co + p * si
    z = torch.stack([zp, zq], -1).flatten(-2) if interleaved else torch.cat([zp, zq], -1)
    return torch.cat([z, y[..., rot:]], -1)
