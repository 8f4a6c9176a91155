"""Windowed attention beside the state rules, and its cache in 4 bits, as measurable cases.

A case is one pass of one operator:

  attn        attention over whole sequences or a segment behind kept keys
  attn_train  a training step of it: forward, and gradients of q, k and v
  store       arriving keys and values written into a cache of 4 bits by pages,
              and a stretch of it read back
  attend      the arriving token(s) of every sequence answered from that cache

Attention, per (sequence, query head) and query t at position p = t + S - T:
  o = sum_j softmax_j(scale q k_j) v_j  over the keys j of p - left .. p + right
  (negative: no bound), zero where there are none; H query heads share HK key heads.

The cache holds an element as sign, two exponent bits and one of mantissa (0, 0.5, 1,
1.5, 2, 3, 4, 6) times a power of two for every 32 elements of a row, the smallest
that leaves them at most 7.  Position p of sequence b is in page
table[b][(p / 64) mod P].  A page is, per key head and with NB = d / 32:
  codes of K   [64 tokens][4 g][NB][4 bytes]      channels 32 blk + 8 g + 2 byte (low half) and + 1
  scales of K  [NB][16 r][4 a]                    token 16 a + r, exponent + 127
  codes of V   [NB][16 pairs][4 g][4 a][4 i]      token 16 a + 4 g + i, channels 32 blk + 2 pair and + 1
  scales of V  [NB][4 g][4 a][4 i]

Inputs: queries, keys and values N(0, 1) per element, logits scaled by d^-1/2.
"""
import math

import torch

own = False

PAGE = 64


# -------------------------------------------------------------------- cases
def _attn(name, kind, B, HK, H, T, d, left=-1, right=0, S=0, io="bf16", layout="bhtd", lengths=False):
    c = dict(kind=kind, B=B, HK=HK, H=H, T=T, S=S or T, d=d, left=left, right=right, io=io,
             layout=layout, lengths=lengths)
    if name:
        c["name"] = name
    return c


def _cache(name, kind, B, HK, H, T, d, held, P, left=-1, back=0, io="bf16", layout="bhtd", lengths=False):
    c = dict(kind=kind, B=B, HK=HK, H=H, T=T, d=d, held=held, P=P, left=left, back=back, io=io,
             layout=layout, lengths=lengths)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a padded batch of short prompts out of a projection's [B, T, H, d] output, grouped heads
        _attn("attn_prompts", "attn", 5, 4, 12, 1000, 64, left=511, layout="bthd", lengths=True),
        # long-context prefill of one prompt in a window
        _attn("attn_32k", "attn", 1, 16, 16, 32768, 64, left=2047),
        # the next segment of a long prompt, behind the keys that its window still sees
        _attn("attn_segment", "attn", 1, 2, 16, 512, 128, left=4095, S=4607),
        # a training step of the 1.3B layer shape, sixteen heads of 64, batch 8
        _attn("train_1p3b", "attn_train", 8, 16, 16, 4096, 64, left=1023, layout="bthd"),
        # sequences of 2k, heads of 128, batch 2, every token before
        _attn("train_d128", "attn_train", 2, 16, 16, 2048, 128),
        # the float32 small-head configuration
        _attn("train_f32", "attn_train", 2, 4, 4, 515, 16, left=127, io="f32"),
        # decode of eight sequences on sixteen heads of 64: the token's row written and given back
        _cache("store_decode", "store", 8, 16, 16, 1, 64, 4096, 65),
        # a whole prompt of 32k written, and read back for the next segment
        _cache("store_32k", "store", 1, 16, 16, 32768, 64, 0, 512),
        # a padded batch behind earlier tokens, in a ring of pages that it runs over
        _cache("store_ring", "store", 5, 4, 12, 1000, 96, 700, 20, back=250, layout="bthd", lengths=True),
        # the same decode's attention, in a window
        _cache("attend_b8_d64", "attend", 8, 16, 16, 1, 64, 4096, 34, left=2047),
        # a full serving batch at head dim 128, four query heads to a key head
        _cache("attend_b64_d128", "attend", 64, 8, 32, 1, 128, 8192, 129),
        # four drafted tokens on a long context
        _cache("attend_draft4", "attend", 4, 4, 16, 4, 128, 65536, 1030),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    while True:
        kind = rng.choice(["attn", "attn", "attn_train", "attn_train", "attn_train", "store", "attend",
                           "attend"])
        io = rng.choice(["bf16"] * 5 + ["f32"])
        layout = rng.choice(["bhtd", "bthd"])
        HK = rng.choice([1, 2, 4, 5, 8, 16])
        H = HK * rng.choice([1, 1, 2, 3, 4, 8] if HK <= 8 else [1, 2])
        lengths = rng.random() < 0.3
        if kind.startswith("attn"):
            d = rng.choice([16, 32, 40, 64, 64, 64, 72, 96, 120, 128, 128])
            B, T = _log_int(rng, 1, 8), _log_int(rng, 1 if rng.random() < 0.1 else 50, 16384)
            left = -1 if rng.random() < 0.3 else _log_int(rng, 1, 4096) - 1
            right = rng.choice([0] * 8 + [-1, 37])
            S = T if rng.random() < 0.7 else T + _log_int(rng, 1, 4096)
            c = _attn(None, kind, B, HK, H, T, d, left, right, S, io, layout, lengths)
            if B * H * T * S <= 3e9 and work(c)["flops"] <= (1e11 if io == "bf16" else 1e10):
                return c
        elif kind == "store":
            d = rng.choice([32, 64, 64, 96, 128])
            T = rng.choice([1, 1, 2, 5]) if rng.random() < 0.4 else _log_int(rng, 20, 16384)
            held, P = rng.choice([0, _log_int(rng, 1, 8192)]), _log_int(rng, 2, 300)
            c = _cache(None, kind, _log_int(rng, 1, 32), HK, H, T, d, held, P, -1,
                       rng.choice([0, 0, _log_int(rng, 1, 2000)]), io, layout, lengths)
            if c["B"] * HK * max(T + c["back"], 64 * P) * d <= 3.3e7:
                return c
        else:
            d, left = rng.choice([32, 64, 64, 96, 128, 128]), -1
            held, T = _log_int(rng, 1, 65536), rng.choice([1, 1, 1, 2, 3, 8])
            P = (held + T) // PAGE + 1 + rng.randint(0, 5)
            if rng.random() < 0.4:           # a ring that holds the window
                left = _log_int(rng, 1, 8192) - 1
                P = min(P, (left + T) // PAGE + 2)
            c = _cache(None, kind, _log_int(rng, 1, 64), HK, H, T, d, held, P, left, 0, io, layout, lengths)
            if c["B"] * HK * 64 * P * d <= 2.6e8 and H * T <= 256:
                return c


def _lengths(c):
    """Live tokens of every sequence: all of the first one's, fewer and fewer behind it."""
    T, B = c["T"], c["B"]
    return [T - T * i // B if c["lengths"] else T for i in range(B)]


def _starts(c):
    """Tokens of every sequence that the cache holds already: between all and half of `held`."""
    return [c["held"] - c["held"] * i // (2 * c["B"]) for i in range(c["B"])]


# ------------------------------------------------------------------- inputs
def _io(c):
    return torch.bfloat16 if c["io"] == "bf16" else torch.float32


def _inputs(c, seed):
    """What the case reads, from the seed alone; token tensors are [B, H, T, d] views."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    B, HK, H, T, d, io = c["B"], c["HK"], c["H"], c["T"], c["d"], _io(c)

    def randn(*s):
        return torch.randn(*s, device=dev, generator=g)

    def rows(heads, tokens):   # the projection's own order in memory behind the same view
        if c["layout"] == "bthd":
            return randn(B, tokens, heads, d).to(io).transpose(1, 2)
        return randn(B, heads, tokens, d).to(io)

    x = {}
    if c["lengths"]:
        x["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device=dev)
    if c["kind"].startswith("attn"):
        x.update(q=rows(H, T), k=rows(HK, c["S"]), v=rows(HK, c["S"]))
        if c["kind"] == "attn_train":
            x["d_out"] = rows(H, T)
        return x
    P = c["P"]
    n = B * P + 3                           # a pool with some free pages
    x["starts"] = torch.tensor(_starts(c), dtype=torch.int32, device=dev)
    x["table"] = torch.randperm(n, device=dev, generator=g)[:B * P].reshape(B, P).to(torch.int32)
    x["cache"] = torch.cat([_pack(randn(m, HK, PAGE, d), randn(m, HK, PAGE, d))
                            for m in [min(1024, n - i) for i in range(0, n, 1024)]])
    if c["kind"] == "store":
        x.update(k=rows(HK, T), v=rows(HK, T))
    else:
        x["q"] = rows(H, T)
    return x


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if case["kind"] == "attn_train":
        for n in ("q", "k", "v"):
            s[n].requires_grad_(True)
    return s


# ------------------------------------------------------------- what is timed
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s)
    if kind == "attn":
        with torch.no_grad():
            return dict(zip(("out", "lse"), _plain_attention(s)))
    if kind == "attn_train":
        out, lse = _plain_attention(s)
        grads = torch.autograd.grad(out, [s["q"], s["k"], s["v"]], s["d_out"])
        return dict(out=out.detach(), lse=lse.detach(), **dict(zip(("d_q", "d_k", "d_v"), grads)))
    if kind == "store":
        return dict(zip(("k", "v"), _plain_store(s)))
    return dict(out=_plain_attend(s))


def _own(s):
    from paper_2608_21308_amd import e2ttt
    c = s["case"]
    io = e2ttt.DT_BF16 if c["io"] == "bf16" else e2ttt.DT_F32
    if "cfg" not in s:      # the handle that a program keeps from call to call
        if c["kind"].startswith("attn"):
            s["cfg"] = e2ttt.AttentionConfig(c["B"], c["HK"], c["H"], c["T"], c["d"], io, S=c["S"],
                                             scale=c["d"] ** -0.5, left=c["left"], right=c["right"])
        else:
            s["cfg"] = e2ttt.CacheConfig(c["B"], c["HK"], c["H"], c["T"], c["d"], c["P"], io,
                                         scale=c["d"] ** -0.5, left=c["left"])
        if c["kind"] == "store":
            s["read"] = e2ttt.CacheConfig(c["B"], c["HK"], c["H"], c["T"] + c["back"], c["d"], c["P"], io)
        if c["kind"] == "attend":
            s["workspace"] = e2ttt.alloc_cache_workspace(s["cfg"])
    cfg, lengths = s["cfg"], s.get("lengths")
    if c["kind"] == "attn":
        return dict(zip(("out", "lse"), e2ttt.attention_forward(cfg, s["q"], s["k"], s["v"],
                                                                lengths=lengths)))
    if c["kind"] == "attn_train":
        out, lse = e2ttt.AttentionFunction.apply(cfg, s["q"], s["k"], s["v"], lengths)
        grads = torch.autograd.grad(out, [s["q"], s["k"], s["v"]], s["d_out"])
        return dict(out=out.detach(), lse=lse.detach(), **dict(zip(("d_q", "d_k", "d_v"), grads)))
    if c["kind"] == "store":
        e2ttt.cache_write(cfg, s["k"], s["v"], s["cache"], s["table"], s["starts"], lengths)
        starts, back = s["starts"], c["back"]
        if back:                # (the stretch begins before the tokens that were written)
            starts, lengths = starts - back, lengths + back if c["lengths"] else None
        return dict(zip(("k", "v"), e2ttt.cache_read(s["read"], s["cache"], s["table"], starts, lengths)))
    return dict(out=e2ttt.cache_attention(cfg, s["q"], s["cache"], s["table"], s["starts"], lengths,
                                          workspace=s["workspace"])[0])


# ------------------------------------------------------------- plain forms
def _plain_attention(s):
    """By blocks of queries, each with the stretch of keys that its bounds reach."""
    c = s["case"]
    T, S, left, right, rep = c["T"], c["S"], c["left"], c["right"], c["H"] // c["HK"]
    q = s["q"].float()
    k, v = (s[n].float().repeat_interleave(rep, 1) for n in ("k", "v"))
    live = s["lengths"] if "lengths" in s else torch.full((c["B"],), T, device=q.device)
    outs, sums = [], []
    for t in range(0, T, 1024):
        n = min(1024, T - t)
        p0 = t + S - T
        lo = 0 if left < 0 else min(max(p0 - left, 0), S - 1)
        hi = S if right < 0 else min(max(p0 + n + right, lo + 1), S)
        p = torch.arange(p0, p0 + n, device=q.device)[:, None]
        j = torch.arange(lo, hi, device=q.device)
        seen = torch.ones(n, hi - lo, dtype=torch.bool, device=q.device)
        if left >= 0:
            seen = seen & (j >= p - left)
        if right >= 0:
            seen = seen & (j <= p + right)
        end = live[:, None, None] + (S - T)
        seen = (seen & (j < end) & (p < end))[:, None]
        x = (q[:, :, t:t + n] @ k[:, :, lo:hi].transpose(-1, -2)) * c["d"] ** -0.5
        x = x.masked_fill(~seen, -math.inf)
        most = x.detach().amax(-1, keepdim=True)
        most = torch.where(most == -math.inf, torch.zeros_like(most), most)
        e = torch.exp(x - most)
        total = e.sum(-1, keepdim=True)
        some = torch.where(total > 0, total, torch.ones_like(total))
        outs.append((e @ v[:, :, lo:hi]) / some)
        sums.append((most + torch.log(total.detach()))[..., 0])
    return torch.cat(outs, 2).to(s["q"].dtype), torch.cat(sums, 2)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """Codes [..., d] (int32) and exponents + 127 [..., d / 32] of rows of floats."""
    y = x.float().unflatten(-1, (-1, 32))
    most = y.abs().amax(-1)
    exp = ((most.view(torch.int32) + 0x1FFFFF) >> 23).sub(2).clamp(2, 254)
    y = torch.ldexp(y, 127 - exp[..., None])
    m = y.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) +
            (m > 5.0) + 8 * torch.signbit(y))
    return code.flatten(-2), exp


def _pairs(code):
    """Two codes to a byte, the even one in the low half."""
    return code[..., 0::2] + 16 * code[..., 1::2]


def _pack(k, v):
    """Pages of bytes from keys and values [..., 64, d]."""
    (kc, ks), (vc, vs) = _quantise(k), _quantise(v)
    nb, n = ks.shape[-1], k.dim() - 2
    kc = _pairs(kc).unflatten(-1, (nb, 4, 4)).transpose(-3, -2)
    ks = ks.unflatten(-2, (4, 16)).movedim(-1, n).transpose(-1, -2)
    vc = _pairs(vc).unflatten(-1, (nb, 16)).unflatten(n, (4, 4, 4)).movedim((-2, -1), (n, n + 1))
    vs = vs.unflatten(n, (4, 4, 4)).movedim(-1, n)
    parts = [kc.flatten(n), ks.flatten(n), vc.transpose(n + 2, n + 3).flatten(n),
             vs.transpose(n + 1, n + 2).flatten(n)]
    return torch.cat([x.to(torch.uint8) for x in parts], -1)


def _unpack(page, d):
    """Keys and values [..., 64, d] in float from pages of bytes [..., 68 d]."""
    nb, n = d // 32, page.dim() - 1
    kc, ks, vc, vs = page.split([32 * d, 2 * d, 32 * d, 2 * d], -1)
    kc = kc.unflatten(-1, (PAGE, 4, nb, 4)).transpose(-3, -2).flatten(-3)
    ks = ks.unflatten(-1, (nb, 16, 4)).transpose(-1, -2).flatten(-2).transpose(-1, -2)
    vc = vc.unflatten(-1, (nb, 16, 4, 4, 4)).transpose(n + 2, n + 3).movedim((n, n + 1), (-2, -1))
    vs = vs.unflatten(-1, (nb, 4, 4, 4)).transpose(n + 1, n + 2).movedim(n, -1)
    grid = torch.tensor(_VALUES, device=page.device)
    grid = torch.cat([grid, -grid])
    table = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)

    def values(code, exp):
        x = table[code.int()].flatten(-2)
        return torch.ldexp(x.unflatten(-1, (nb, 32)), exp.int()[..., None] - 127).flatten(-2)

    return (values(kc, ks),
            values(vc.flatten(n, n + 2).flatten(-2), vs.flatten(n, n + 2)))


def _place(s, p):
    """Pages and rows in them of positions p [B, n]."""
    page = s["table"].long().gather(1, torch.div(p, PAGE, rounding_mode="floor") % s["case"]["P"])
    return page, p % PAGE


def _ends(s):
    """Tokens of every sequence once the arriving ones are written."""
    c = s["case"]
    return s["starts"].long() + (s["lengths"].long() if c["lengths"] else c["T"])


def _plain_store(s):
    c = s["case"]
    T, P, d, dev = c["T"], c["P"], c["d"], s["k"].device
    t = torch.arange(T, device=dev)
    p, end = s["starts"].long()[:, None] + t, _ends(s)[:, None]
    first = ((end - 1) // PAGE - P + 1) * PAGE          # what the ring still holds
    b, t = torch.nonzero((p < end) & (p >= first), as_tuple=True)
    page, row = _place(s, p)
    page, row = page[b, t], row[b, t]
    cache = s["cache"]
    (kc, ks), (vc, vs) = (_quantise(s[n][b, :, t]) for n in ("k", "v"))    # [tokens, HK, ..]
    nb, h = d // 32, torch.arange(c["HK"], device=dev)[:, None, None]
    blk, i = torch.arange(nb, device=dev)[:, None], torch.arange(16, device=dev)

    def put(at, x):
        at = at + torch.zeros_like(x)
        cache[page[:, None, None, None].expand_as(at), (h + torch.zeros_like(x)), at] = x.to(torch.uint8)

    r = row[:, None, None, None]
    put(r * 16 * nb + (i // 4) * 4 * nb + blk * 4 + i % 4, _pairs(kc).unflatten(-1, (nb, 16)).long())
    put(32 * d + blk * 64 + (r % 16) * 4 + r // 16, ks[..., None].long())
    at = (r // 4 % 4) * 16 + (r // 16) * 4 + r % 4
    put(34 * d + (blk * 16 + i) * 64 + at, _pairs(vc).unflatten(-1, (nb, 16)).long())
    put(66 * d + blk * 64 + at, vs[..., None].long())

    # the stretch that is read back, row by row
    p = s["starts"].long()[:, None] - c["back"] + torch.arange(T + c["back"], device=dev)
    some = ((p >= 0) & (p >= first) & (p < end))[:, None, :, None]
    page, row = _place(s, p.clamp(min=0))
    k, v = _unpack(cache[s["table"].long()], d)          # [B, P, HK, 64, d]
    at = (p.clamp(min=0) // PAGE % P) * PAGE + row

    def rows(x):
        x = x.transpose(1, 2).flatten(2, 3)
        x = x.gather(2, at[:, None, :, None].expand(-1, c["HK"], -1, d))
        return torch.where(some, x, torch.zeros_like(x)).to(_io(c))

    return rows(k), rows(v)


def _plain_attend(s):
    c = s["case"]
    B, HK, T, P, d, rep = c["B"], c["HK"], c["T"], c["P"], c["d"], c["H"] // c["HK"]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _unpack(s["cache"][s["table"].long()], d))
    dev, end = k.device, _ends(s)[:, None]
    last = (end - 1) // PAGE
    page = last - (last - torch.arange(P, device=dev)) % P         # what each entry holds now
    j = (page[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(1)[:, None]
    p = (s["starts"].long()[:, None] + torch.arange(T, device=dev))[..., None]
    seen = (j >= 0) & (j <= p) & (p < end[..., None])
    if c["left"] >= 0:
        seen = seen & (j >= p - c["left"])
    q = s["q"].float().unflatten(1, (HK, rep)).flatten(2, 3)       # rep x T queries of a key head
    seen = seen[:, None, None].expand(B, 1, rep, T, P * PAGE).flatten(2, 3)
    x = ((q @ k.transpose(-1, -2)) * d ** -0.5).masked_fill(~seen, -math.inf)
    most = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(most == -math.inf, torch.zeros_like(most), most))
    total = e.sum(-1, keepdim=True)
    o = (e @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.unflatten(2, (rep, T)).flatten(1, 2).to(s["q"].dtype)


# ------------------------------------------------------------ what it costs
def _sees(c):
    """Pairs of a query and a key that it sees, and keys that some query sees, per head."""
    off, pairs, keys = c["S"] - c["T"], 0, 0
    for n in _lengths(c):
        end = n + off

        def upto(m):        # sum over positions p < m of min(p + right + 1, end)
            if c["right"] < 0:
                return end * m
            full = max(0, min(m, end - c["right"]))
            return full * (full - 1) // 2 + full * (c["right"] + 1) + (m - full) * end

        pairs += upto(end) - upto(off)
        if c["left"] >= 0:  # keys j < p - left
            a, b = max(0, off - c["left"]), max(0, end - c["left"])
            pairs -= b * (b - 1) // 2 - a * (a - 1) // 2
        if n:
            keys += end - (0 if c["left"] < 0 else max(0, off - c["left"]))
    return pairs, keys


def work(c):
    """Inputs read once, outputs written once. Forward: two products for every pair that is seen;
    backward: five (the probabilities formed again)."""
    e, B, HK, H, T, d = 2 if c["io"] == "bf16" else 4, c["B"], c["HK"], c["H"], c["T"], c["d"]
    live, row = sum(_lengths(c)), d // 2 + d // 32
    if c["kind"].startswith("attn"):
        pairs, keys = _sees(c)
        fwd = {"bytes": (live + B * T) * H * d * e + 2 * keys * HK * d * e + 4 * B * H * T,
               "flops": 4.0 * d * H * pairs}
        if c["kind"] == "attn":
            return fwd
        return {"bytes": fwd["bytes"] + (live + B * T) * H * d * e + 2 * B * c["S"] * HK * d * e,
                "flops": 14.0 * d * H * pairs}
    if c["kind"] == "store":
        given, back = live * HK * d, B * (T + c["back"]) * HK * d
        held = sum(min(n + c["back"], 64 * c["P"], s + n) for n, s in zip(_lengths(c), _starts(c)))
        return {"bytes": 2 * (given + back) * e + 2 * HK * row * (live + held), "flops": 8 * (given + back)}
    seen = pairs = 0
    for n, s in zip(_lengths(c), _starts(c)):
        if n:
            w = s + n if c["left"] < 0 else min(s + n, c["left"] + n)
            w = min(w, 64 * c["P"])
            seen, pairs = seen + w, pairs + n * (w - n / 2)
    return {"bytes": 2 * seen * HK * row + (live + B * T) * H * d * e, "flops": 4.0 * d * H * pairs}


# ------------------------------------------------------------ in 64 bits
def exact(c, seed):
    x = _inputs(c, seed)
    return {"attn": _exact_attention, "attn_train": _exact_attention, "store": _exact_store,
            "attend": _exact_attend}[c["kind"]](c, x)


def _exact_attention(c, x):
    """Sequence by sequence and head by head: the live keys' softmax and its derivative."""
    B, HK, H, T, S, d = c["B"], c["HK"], c["H"], c["T"], c["S"], c["d"]
    train, sc = c["kind"] == "attn_train", c["d"] ** -0.5
    dev, rep = x["q"].device, H // HK
    got = dict(out=torch.zeros(B, H, T, d, dtype=torch.float64, device=dev),
               lse=torch.full((B, H, T), -math.inf, dtype=torch.float64, device=dev))
    if train:
        got["d_q"] = torch.zeros_like(got["out"])
        got["d_k"], got["d_v"] = (torch.zeros(B, HK, S, d, dtype=torch.float64, device=dev) for _ in "kv")
    step = 2048
    for b, n in enumerate(_lengths(c)):
        end = n + S - T
        for h in range(HK):
            qs = slice(h * rep, (h + 1) * rep)
            for t in range(0, n, step):
                m = min(step, n - t)
                pos = torch.arange(t, t + m, device=dev) + (S - T)
                a = max(0, t + S - T - c["left"]) if c["left"] >= 0 else 0
                z = min(end, t + m + S - T + c["right"]) if c["right"] >= 0 else end
                if z <= a:
                    continue
                k, v = x["k"][b, h, a:z].double(), x["v"][b, h, a:z].double()
                q = x["q"][b, qs, t:t + m].double()
                far = torch.arange(a, z, device=dev)[None, :] - pos[:, None]
                hide = torch.zeros_like(far, dtype=torch.bool)
                if c["left"] >= 0:
                    hide |= far < -c["left"]
                if c["right"] >= 0:
                    hide |= far > c["right"]
                z_ = torch.matmul(q, k.t()).mul_(sc).masked_fill_(hide, -math.inf)
                lse = torch.logsumexp(z_, -1)
                w = torch.exp(z_ - torch.where(lse == -math.inf, 0.0, lse)[..., None])
                o = torch.matmul(w, v)
                got["out"][b, qs, t:t + m], got["lse"][b, qs, t:t + m] = o, lse
                if train:
                    g = x["d_out"][b, qs, t:t + m].double()
                    got["d_v"][b, h, a:z] += torch.matmul(w.transpose(-1, -2), g).sum(0)
                    w *= torch.matmul(g, v.t()) - (g * o).sum(-1, keepdim=True)
                    got["d_q"][b, qs, t:t + m] = torch.matmul(w, k) * sc
                    got["d_k"][b, h, a:z] += torch.matmul(w.transpose(-1, -2), q).sum(0) * sc
    return got


def _row(c, cache, page, j, what):
    """Rows j of pages [n] of `what` ("k" or "v"), every key head, [n, HK, d] in 64 bits: byte
    by byte from the layout."""
    d, dev = c["d"], cache.device
    nb, ch = d // 32, torch.arange(d, device=dev)
    blk, j = ch // 32, j[:, None]
    if what == "k":
        code = j * (16 * nb) + (ch % 32 // 8) * (4 * nb) + blk * 4 + ch % 8 // 2
        scale = 32 * d + blk * 64 + (j % 16) * 4 + j // 16
    else:
        at = (j % 16 // 4) * 16 + (j // 16) * 4 + j % 4
        code = 34 * d + (ch // 2) * 64 + at
        scale = 66 * d + blk * 64 + at
    heads = torch.arange(c["HK"], device=dev)[None, :, None]
    byte = cache[page[:, None, None], heads, code[:, None]].int()
    bits = torch.where(ch % 2 == 1, byte >> 4, byte & 15)
    e, m = (bits >> 1 & 3).double(), (bits & 1).double()
    mag = torch.where(e == 0, 0.5 * m, torch.exp2(e - 1) * (1 + 0.5 * m))
    power = cache[page[:, None, None], heads, scale[:, None]].double() - 127
    return torch.where(bits >= 8, -mag, mag) * torch.exp2(power)


def _nearest(x):
    """Rows as the cache gives them back."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    mant, power = torch.frexp(top / 7.0)
    power = torch.where(mant == 0.5, power - 1, power).clamp(-125, 127).double()
    y = y / torch.exp2(power)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((torch.round(y / step) * step).clamp(-6, 6) * torch.exp2(power)).flatten(-2)


def _exact_store(c, x):
    B, HK, T, P, d, back = c["B"], c["HK"], c["T"], c["P"], c["d"], c["back"]
    dev, table = x["k"].device, x["table"].long()
    got = {n: torch.zeros(B, HK, T + back, d, dtype=torch.float64, device=dev) for n in ("k", "v")}
    for b, (n, s) in enumerate(zip(_lengths(c), _starts(c))):
        end = s + n
        p = torch.arange(max(0, s - back, ((end - 1) // PAGE - P + 1) * PAGE), end, device=dev)
        for what in ("k", "v"):
            old, new = p[p < s], p[p >= s]
            rows = [_row(c, x["cache"], table[b, old // PAGE % P], old % PAGE, what).transpose(0, 1),
                    _nearest(x[what][b, :, new - s])]
            got[what][b, :, p - (s - back)] = torch.cat(rows, 1)
    return got


def _exact_attend(c, x):
    B, HK, H, T, P, d = c["B"], c["HK"], c["H"], c["T"], c["P"], c["d"]
    rep, dev, table = H // HK, x["q"].device, x["table"].long()
    got = torch.zeros(B, H, T, d, dtype=torch.float64, device=dev)
    for b, (n, s) in enumerate(zip(_lengths(c), _starts(c))):
        if not n:
            continue
        a = max(0, ((s + n - 1) // PAGE - P + 1) * PAGE, s - c["left"] if c["left"] >= 0 else 0)
        j = torch.arange(a, s + n, device=dev)
        k, v = (_row(c, x["cache"], table[b, j // PAGE % P], j % PAGE, w).transpose(0, 1) for w in "kv")
        q = x["q"][b, :, :n].double().reshape(HK, rep * n, d)
        z = torch.matmul(q, k.transpose(-1, -2)) * d ** -0.5
        far = (j[None, :] - torch.arange(s, s + n, device=dev)[:, None]).repeat(rep, 1)
        hide = far > 0
        if c["left"] >= 0:
            hide |= far < -c["left"]
        z = z.masked_fill(hide, -math.inf)
        w = torch.exp(z - torch.logsumexp(z, -1, keepdim=True).clamp(min=-1e300))
        got[b, :, :n] = torch.matmul(w, v).reshape(H, n, d)
    return dict(out=got)
