"""Token-mixing operators next to the chunk update, as measurable cases.

A case is one pass of one operator:

  step     recurrent decode of the gated delta rule: the arriving token(s) of
           every sequence update its state and are answered from it
  prefill  the gated delta rule over whole prompts, from a state to a state
  train    a training step of that rule: forward, and gradients of every input
  qk       query/key preparation (SiLU, unit length, rotary positions)
  qk_train its forward and backward

The rule, per (sequence, value head) and token, with a state W [dv][dk]:
  W <- exp(g) W;  e = v - W k;  W <- W + eta e k^T;  o = scale W q.

Inputs: queries and keys of unit length, values that a head can learn (a
per-head linear map of the key plus noise), learning rates sigmoid(N(0, 1)),
log decays -a softplus(N(0, 1) + c) with a rate a per head as such layers are
initialised, and a running state of the size such decays leave.
"""
import math

import torch

own = False


# -------------------------------------------------------------------- cases
def _case(name, kind, B, HK, H, T, dk, dv, io="bf16", layout="bhtd", lengths=False, decay=True):
    c = dict(kind=kind, B=B, HK=HK, H=H, T=T, dk=dk, dv=dv, io=io, layout=layout,
             lengths=lengths, decay=decay)
    if name:
        c["name"] = name
    return c


def _qk(name, kind, B, HK, H, T, d, rot, io="bf16", layout="bhtd", interleaved=False,
        silu=True, unit=True, factor=1.0, far=0):
    c = dict(kind=kind, B=B, HK=HK, H=H, T=T, d=d, rot=rot, io=io, layout=layout,
             interleaved=interleaved, silu=silu, unit=unit, factor=factor, far=far)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # decode of eight sequences on sixteen heads of 64: the call made for every token
        _case("step_b8_d64", "step", 8, 16, 16, 1, 64, 64),
        # a full serving batch at head dim 128, two value heads to a key head, states in a pool
        _case("step_b128_d128", "step", 128, 16, 32, 1, 128, 128),
        # four drafted tokens of sixteen sequences at once
        _case("step_draft4", "step", 16, 16, 16, 4, 128, 128),
        # prefill of two 2k prompts on four heads (a tensor-parallel slice)
        _case("prefill_b2h4", "prefill", 2, 4, 4, 2048, 64, 64),
        # long-context prefill of one prompt
        _case("prefill_32k", "prefill", 1, 16, 16, 32768, 128, 128),
        # a padded batch of short prompts out of a projection's [B, T, H, d] output
        _case("prefill_ragged", "prefill", 5, 4, 12, 1000, 64, 120, layout="bthd", lengths=True),
        # a training step of the 1.3B layer shape, sixteen heads of 64, batch 8
        _case("train_1p3b", "train", 8, 16, 16, 4096, 64, 64),
        # sequences of 2k, heads of 128, batch 2
        _case("train_d128", "train", 2, 16, 16, 2048, 128, 128, layout="bthd"),
        # the float32 small-head configuration
        _case("train_f32", "train", 2, 4, 4, 515, 16, 16, io="f32"),
        # decode's query/key preparation, far into a context scaled to four times its length
        _qk("qk_decode", "qk", 8, 16, 16, 1, 64, 64, factor=4.0, far=30000),
        # the training step's preparation at the 1.3B layer shape
        _qk("qk_train_1p3b", "qk_train", 8, 16, 16, 4096, 64, 64, layout="bthd"),
        # part of the head, interleaved pairs, grouped keys, an odd length
        _qk("qk_train_part", "qk_train", 1, 4, 16, 1501, 128, 48, interleaved=True, silu=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["step", "prefill", "prefill", "train", "train", "qk", "qk_train"])
    io = rng.choice(["bf16"] * 5 + ["f32"])
    layout = rng.choice(["bhtd", "bthd"])
    HK = rng.choice([1, 2, 4, 5, 8, 16])
    H = HK * rng.choice([1, 1, 2, 3] if HK <= 8 else [1, 2])
    if kind.startswith("qk"):
        d = rng.choice([16, 32, 64, 64, 72, 96, 128, 128])
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)])
        B = _log_int(rng, 1, 32)
        T = rng.choice([1, 1, 2, 5]) if kind == "qk" else _log_int(rng, 20, 500000 // (B * H))
        return _qk(None, kind, B, HK, H, T, d, rot, io, layout, rng.random() < 0.4,
                   rng.random() < 0.7, rng.random() < 0.7, rng.choice([1.0, 1.0, 4.0, 7.5]),
                   rng.choice([0, 1000, 100000]))
    dk = rng.choice([16, 32, 64, 64, 64, 72, 128, 128])
    dv = rng.choice([dk, dk, dk, 24, 64, 120, 128, 192])
    decay = rng.random() < 0.9
    if kind == "step":
        return _case(None, kind, _log_int(rng, 1, 96), HK, H, rng.choice([1, 1, 1, 2, 3, 8]),
                     dk, dv, io, layout, False, decay)
    B = _log_int(rng, 1, 8)
    most = min(8192 if kind == "prefill" else 4096, 400000 // (B * H))
    if io == "f32":
        most = min(most, 2048)
    T = rng.randint(1, 64) if rng.random() < 0.15 else _log_int(rng, 65, most)
    return _case(None, kind, B, HK, H, T, dk, dv, io, layout, rng.random() < 0.3, decay)


# ------------------------------------------------------------------- inputs
def _frequencies(c):
    """Rotary frequencies at base 10000; a context stretched by `factor` scales
    the base (so the lowest frequency falls by about the factor)."""
    base = 10000.0 * c["factor"] ** (c["rot"] / max(1.0, c["rot"] - 2.0))
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64)
    return (base ** (-i / c["rot"])).float()


def _rot_scale(c):
    return 0.1 * math.log(c["factor"]) + 1.0


def _inputs(c, seed):
    """What the case reads, from the seed alone; token tensors are [B, H, T, d] views."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    B, HK, H, T = c["B"], c["HK"], c["H"], c["T"]
    io = torch.bfloat16 if c["io"] == "bf16" else torch.float32

    def randn(*s):
        return torch.randn(*s, device=dev, generator=g)

    def lay(x):       # the projection's own order in memory behind the same view
        return x.transpose(1, 2).contiguous().transpose(1, 2) if c["layout"] == "bthd" else x

    def unit(x):
        return x / x.norm(dim=-1, keepdim=True)

    if c["kind"].startswith("qk"):
        x = dict(q=lay(randn(B, H, T, c["d"]).to(io)), k=lay(randn(B, HK, T, c["d"]).to(io)))
        x["inv_freq"] = _frequencies(c).to(dev)
        first = torch.randint(0, c["far"] + 1, (B, 1), device=dev, generator=g)
        x["positions"] = (first + torch.arange(T, device=dev)).contiguous()
        if c["kind"] == "qk_train":
            x["d_q"], x["d_k"] = lay(randn(B, H, T, c["d"]).to(io)), lay(randn(B, HK, T, c["d"]).to(io))
        return x
    dk, dv = c["dk"], c["dv"]
    x = dict(q=lay(unit(randn(B, HK, T, dk)).to(io)), k=lay(unit(randn(B, HK, T, dk)).to(io)))
    kh = x["k"].float().repeat_interleave(H // HK, 1)
    x["v"] = lay((0.8 * torch.matmul(kh, randn(H, dk, dv)) + 0.6 * randn(B, H, T, dv)).to(io))
    x["eta"] = lay(torch.sigmoid(randn(B, H, T, 1)))[..., 0]
    if c["decay"]:
        rate = torch.exp(math.log(16.0) * torch.rand(H, 1, 1, device=dev, generator=g))
        x["log_gamma"] = lay(-rate * torch.nn.functional.softplus(randn(B, H, T, 1) - 4.5))[..., 0]
    if c["kind"] == "step":
        n = B + B // 4 + 1          # a pool with some free slots
        x["w"] = 0.3 * randn(n, H, dv, dk)
        x["slots"] = torch.randperm(n, device=dev, generator=g)[:B].to(torch.int32)
        return x
    x["w_in"] = 0.3 * randn(B, H, dv, dk)
    if c["lengths"]:
        x["lengths"] = torch.randint(0, T + 1, (B,), device=dev, generator=g).to(torch.int32)
        x["lengths"][0] = T
    if c["kind"] == "train":
        x["d_out"], x["d_w_out"] = lay(randn(B, H, T, dv).to(io)), 0.1 * randn(B, H, dv, dk)
    return x


_LEAVES = ("q", "k", "v", "eta", "log_gamma", "w_in")


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["kind"].endswith("train"):
        for n in _LEAVES if case["kind"] == "train" else ("q", "k"):
            if n in s:
                s[n].requires_grad_(True)
    return s


# ------------------------------------------------------------- what is timed
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s)
    if kind == "step":
        return _plain_step(s)
    if kind == "prefill":
        with torch.no_grad():
            return dict(zip(("out", "w_out"), _plain_delta(s)))
    if kind == "train":
        out, w_out = _plain_delta(s)
        names = [n for n in _LEAVES if n in s]
        grads = torch.autograd.grad([out, w_out], [s[n] for n in names], [s["d_out"], s["d_w_out"]])
        return dict(out=out.detach(), w_out=w_out.detach(),
                    **{"d_" + n: x for n, x in zip(names, grads)})
    if kind == "qk":
        return dict(zip(("q", "k"), _plain_qk(s)))
    q, k = _plain_qk(s)
    dq, dk = torch.autograd.grad([q, k], [s["q"], s["k"]], [s["d_q"], s["d_k"]])
    return dict(q=q.detach(), k=k.detach(), d_q=dq, d_k=dk)


def _own(s):
    from paper_2608_21308_amd import e2ttt
    c = s["case"]
    if "cfg" not in s:      # the handle and buffers that a program keeps from call to call
        io = e2ttt.DT_BF16 if c["io"] == "bf16" else e2ttt.DT_F32
        if c["kind"].startswith("qk"):
            flags = ((e2ttt.QK_SILU if c["silu"] else 0) | (e2ttt.QK_UNIT if c["unit"] else 0) |
                     (e2ttt.QK_INTERLEAVED if c["interleaved"] else 0))
            s["cfg"] = e2ttt.QKConfig(c["B"], c["H"], c["HK"], c["T"], c["d"], c["rot"], io, flags,
                                      rot_scale=_rot_scale(c))
        else:
            s["cfg"] = e2ttt.DeltaConfig(c["B"], c["HK"], c["H"], c["T"], c["dk"], c["dv"], io,
                                         scale=c["dk"] ** -0.5)
        if c["kind"] == "prefill":
            s["workspace"] = e2ttt.alloc_delta_workspace(s["cfg"], False)
    cfg, gam = s["cfg"], s.get("log_gamma")
    if c["kind"] == "step":
        out = e2ttt.delta_step(cfg, s["q"], s["k"], s["v"], s["eta"], gam, s["w"], slots=s["slots"])
        return dict(out=out, w=s["w"])
    if c["kind"] == "prefill":
        out, w_out, _ = e2ttt.delta_forward(cfg, s["q"], s["k"], s["v"], s["eta"], gam, s["w_in"],
                                            lengths=s.get("lengths"), workspace=s["workspace"])
        return dict(out=out, w_out=w_out)
    if c["kind"] == "train":
        out, w_out = e2ttt.DeltaFunction.apply(cfg, s["q"], s["k"], s["v"], s["eta"], gam,
                                               s["w_in"], s.get("lengths"))
        names = [n for n in _LEAVES if n in s]
        grads = torch.autograd.grad([out, w_out], [s[n] for n in names], [s["d_out"], s["d_w_out"]])
        return dict(out=out.detach(), w_out=w_out.detach(),
                    **{"d_" + n: x for n, x in zip(names, grads)})
    if c["kind"] == "qk":
        return dict(zip(("q", "k"), e2ttt.qk_forward(cfg, s["q"], s["k"], s["inv_freq"],
                                                     s["positions"])))
    q, k = e2ttt.QKFunction.apply(cfg, s["q"], s["k"], s["inv_freq"], s["positions"])
    dq, dk = torch.autograd.grad([q, k], [s["q"], s["k"]], [s["d_q"], s["d_k"]])
    return dict(q=q.detach(), k=k.detach(), d_q=dq, d_k=dk)


# ------------------------------------------------------------- plain forms
def _repeat(x, c):
    return x.float().repeat_interleave(c["H"] // c["HK"], 1)


def _plain_step(s):
    """Token by token at the states of the batch's slots."""
    c, slots = s["case"], s["slots"].long()
    w = s["w"][slots]
    q, k, v = _repeat(s["q"], c), _repeat(s["k"], c), s["v"].float()
    outs = []
    for t in range(c["T"]):
        kt = k[:, :, t, :, None]
        if c["decay"]:
            w = w * torch.exp(s["log_gamma"][:, :, t])[..., None, None]
        u = (v[:, :, t, :, None] - w @ kt) * s["eta"][:, :, t, None, None]
        w = w + u * kt.transpose(-1, -2)
        outs.append((w @ q[:, :, t, :, None])[..., 0] * c["dk"] ** -0.5)
    s["w"][slots] = w
    return dict(out=torch.stack(outs, 2).to(s["q"].dtype), w=s["w"])


def _unit_lower_inverse(a):
    """(I + a)^-1 of strictly lower triangular a, by blocks of doubling size:
    the inverse of [[X, 0], [Z, Y]] has -Y^-1 Z X^-1 below its diagonal blocks."""
    n = a.shape[-1]
    inv = torch.eye(n, device=a.device, dtype=a.dtype).expand(a.shape)
    half = 1
    while half < n:
        i = torch.arange(n, device=a.device)
        below = (i[:, None] // half == i[None, :] // half + 1) & (i[:, None] // half % 2 == 1)
        inv = inv - inv @ (a * below) @ inv
        half *= 2
    return inv


def _plain_delta(s):
    """The rule in its chunked form: within a chunk of 64 tokens the updates solve a
    triangular system, between chunks only the state is carried."""
    c = s["case"]
    B, H, T, dk, dv, C = c["B"], c["H"], c["T"], c["dk"], c["dv"], 64
    q, k, v = _repeat(s["q"], c) * dk ** -0.5, _repeat(s["k"], c), s["v"].float()
    eta = s["eta"]
    gam = s["log_gamma"] if c["decay"] else torch.zeros_like(eta)
    if "lengths" in s:
        live = torch.arange(T, device=eta.device) < s["lengths"][:, None, None]
        q, k, v = q * live[..., None], k * live[..., None], v * live[..., None]
        eta, gam = eta * live, gam * live
    n = (T + C - 1) // C
    pad = n * C - T

    def chunks(x):
        x = torch.nn.functional.pad(x, (0, 0, 0, pad) if x.dim() == 4 else (0, pad))
        return x.reshape(B, H, n, C, *x.shape[3:])

    q, k, v, eta, gam = (chunks(x) for x in (q, k, v, eta, gam))
    b = gam.double().cumsum(-1)
    ones = torch.ones(C, C, device=q.device)
    low = torch.where(ones.tril() > 0, b[..., :, None] - b[..., None, :],
                      b.new_full((), -math.inf)).exp().float()
    inner = (low * (k @ k.transpose(-1, -2))).tril(-1)
    inv = _unit_lower_inverse(eta[..., None] * inner)
    attn = low * (q @ k.transpose(-1, -2))
    from_start, to_end = b.exp().float(), (b[..., -1:] - b).exp().float()
    k_start, q_start = k * from_start[..., None], q * from_start[..., None]
    k_end, solve = k * to_end[..., None], inv * eta[..., None, :]
    w, outs = s["w_in"], []
    for r in range(n):
        u = solve[:, :, r] @ (v[:, :, r] - k_start[:, :, r] @ w.transpose(-1, -2))
        outs.append(q_start[:, :, r] @ w.transpose(-1, -2) + attn[:, :, r] @ u)
        w = w * from_start[:, :, r, -1, None, None] + u.transpose(-1, -2) @ k_end[:, :, r]
    return torch.cat(outs, 2)[:, :, :T].to(s["q"].dtype), w


def _plain_qk(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = s["positions"][:, None, :, None].double() * s["inv_freq"].double()
    cos, sin = (torch.cos(angle) * _rot_scale(c)).float(), (torch.sin(angle) * _rot_scale(c)).float()

    def one(x):
        y = x.float()
        if c["silu"]:
            y = y / (1.0 + torch.exp(-y))
        if c["unit"]:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) + 1e-6)
        if c["interleaved"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = y[..., :half], y[..., half:rot]
            z = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([z, y[..., rot:]], -1).to(x.dtype)

    return one(s["q"]), one(s["k"])


# ------------------------------------------------------------ what it costs
def work(c):
    """Inputs read once, outputs written once. A token of the rule takes three products with
    the state (W k, e k^T, W q); its backward eight (two of them the state formed again)."""
    e = 2 if c["io"] == "bf16" else 4
    if c["kind"].startswith("qk"):
        n = c["B"] * (c["H"] + c["HK"]) * c["T"] * c["d"]
        if c["kind"] == "qk":
            return {"bytes": 2 * n * e, "flops": 12 * n}
        return {"bytes": 4 * n * e, "flops": 36 * n}
    B, HK, H, T, dk, dv = c["B"], c["HK"], c["H"], c["T"], c["dk"], c["dv"]
    rows = B * T * (2 * HK * dk + 2 * H * dv) * e
    gates = B * H * T * (8 if c["decay"] else 4)
    state, unit = B * H * dk * dv * 4, 2.0 * B * H * T * dk * dv
    if c["kind"] != "train":
        return {"bytes": rows + gates + 2 * state, "flops": 3 * unit}
    return {"bytes": 2 * rows + 2 * gates + 4 * state, "flops": 11 * unit}


# ------------------------------------------------------------ in 64 bits
def exact(c, seed):
    x = {n: t.double() if t.is_floating_point() else t for n, t in _inputs(c, seed).items()}
    if c["kind"].startswith("qk"):
        return _exact_qk(c, x)
    return _exact_delta(c, x)


def _exact_qk(c, x):
    """Rotations as products of complex numbers; gradients by the transposed map."""
    rot, ph = c["rot"], x["positions"][:, None, :, None].double() * x["inv_freq"]
    turn = torch.polar(torch.full_like(ph, _rot_scale(c)), ph)

    def pairs(y):
        y = y[..., :rot]
        y = y.unflatten(-1, (-1, 2)) if c["interleaved"] else y.unflatten(-1, (2, -1)).transpose(-1, -2)
        return torch.view_as_complex(y.contiguous())

    def flat(z):
        z = torch.view_as_real(z)
        return z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)

    def turned(y, by):
        return torch.cat([flat(pairs(y) * by), y[..., rot:]], -1)

    out = {}
    for n in ("q", "k"):
        sg = torch.sigmoid(x[n])
        y = x[n] * sg if c["silu"] else x[n]
        r = (y.square().sum(-1, keepdim=True) + 1e-6).rsqrt() if c["unit"] else torch.ones_like(y[..., :1])
        out[n] = turned(y * r, turn)
        if c["kind"] == "qk_train":
            d = turned(x["d_" + n], turn.conj())
            d = r * (d - y * r * r * (y * d).sum(-1, keepdim=True)) if c["unit"] else d
            out["d_" + n] = d * sg * (1 + x[n] * (1 - sg)) if c["silu"] else d
    return out


def _exact_delta(c, x):
    """The recurrence itself, token by token, and its adjoint in reverse over stretches of
    64 tokens whose states are formed again."""
    B, HK, H, T, dk, dv = c["B"], c["HK"], c["H"], c["T"], c["dk"], c["dv"]
    rep, sc = H // HK, dk ** -0.5
    q, k = x["q"].repeat_interleave(rep, 1), x["k"].repeat_interleave(rep, 1)
    v, eta = x["v"], x["eta"]
    gam = x["log_gamma"].exp() if c["decay"] else torch.ones_like(eta)
    if "lengths" in x:
        dead = torch.arange(T, device=eta.device) >= x["lengths"][:, None, None]
        q, k, v = (y.masked_fill(dead[..., None], 0.0) for y in (q, k, v))
        eta, gam = eta.masked_fill(dead, 0.0), gam.masked_fill(dead, 1.0)
    w = x["w"][x["slots"].long()] if c["kind"] == "step" else x["w_in"]
    out, starts = torch.empty_like(v), []

    def token(w, t):
        wd = w * gam[:, :, t, None, None]
        e = v[:, :, t] - (wd @ k[:, :, t, :, None])[..., 0]
        u = e * eta[:, :, t, None]
        return wd, e, u, wd + u[..., None] * k[:, :, t, None, :]

    for t in range(T):
        if t % 64 == 0:
            starts.append(w)
        w = token(w, t)[3]
        out[:, :, t] = (w @ q[:, :, t, :, None])[..., 0] * sc
    if c["kind"] == "step":
        x["w"][x["slots"].long()] = w
        return dict(out=out, w=x["w"])
    if c["kind"] == "prefill":
        return dict(out=out, w_out=w)
    w_out, dw, do = w, x["d_w_out"].clone(), x["d_out"] * sc
    if "lengths" in x:
        do = do.masked_fill(dead[..., None], 0.0)
    dq, dkk, d_v = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    d_eta, d_gam = torch.empty_like(eta), torch.empty_like(eta)
    for i in reversed(range(len(starts))):
        w, kept = starts[i], []
        for t in range(64 * i, min(T, 64 * i + 64)):
            kept.append(token(w, t))
            w = kept[-1][3]
        for t in reversed(range(64 * i, min(T, 64 * i + 64))):
            wd, e, u, w = kept.pop()
            dw = dw + do[:, :, t, :, None] * q[:, :, t, None, :]
            dq[:, :, t] = (do[:, :, t, None, :] @ w)[..., 0, :]
            du = (dw @ k[:, :, t, :, None])[..., 0]
            d_eta[:, :, t] = (du * e).sum(-1)
            de = du * eta[:, :, t, None]
            d_v[:, :, t] = de
            dkk[:, :, t] = (u[..., None, :] @ dw - de[..., None, :] @ wd)[..., 0, :]
            dw = dw - de[..., None] * k[:, :, t, None, :]
            d_gam[:, :, t] = (dw * wd).sum((-1, -2))
            dw = dw * gam[:, :, t, None, None]
    if "lengths" in x:
        dq, dkk, d_v = (y.masked_fill(dead[..., None], 0.0) for y in (dq, dkk, d_v))
        d_eta, d_gam = d_eta.masked_fill(dead, 0.0), d_gam.masked_fill(dead, 0.0)
    got = dict(out=out, w_out=w_out, d_q=dq.unflatten(1, (HK, rep)).sum(2),
               d_k=dkk.unflatten(1, (HK, rep)).sum(2), d_v=d_v, d_eta=d_eta, d_w_in=dw)
    if c["decay"]:
        got["d_log_gamma"] = d_gam
    return got
