"""GPU parity of attention and its gradients with 64 bits (tests/attnref.py),
element by element within the bounds derived there, and in the 2-norm: with bf16
a result passes two roundings of rms at most 2^-8 / sqrt(3) each (its operand's,
its own), so 2^-8 of the whole; a gradient of queries or keys a third one, of the
out that D is formed from: 1.5 2^-8.  With float32 the errors behind the
elements' bounds have either sign: 2^-18."""
import dataclasses
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import attnref
from tests.test_gpu_delta import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def rounded(x, io):
    return x.to(torch.bfloat16 if io == "bf16" else torch.float32).double()


def inputs(B, HK, H, T, S, d, io, seed, lengths=None, size=1.0):
    """q, k, v, d_out in float64 at the io type's values; what is not live is NaN."""
    g = torch.Generator().manual_seed(seed)
    rn = lambda h, t: rounded(size * torch.randn(B, h, t, d, generator=g, dtype=torch.float64), io)
    x = dict(q=rn(H, T), k=rn(HK, S), v=rn(HK, S))
    d_out = rn(H, T)
    if lengths is not None:
        for b, n in enumerate(lengths.clamp(0, T).tolist()):
            x["q"][b, :, n:] = math.nan
            d_out[b, :, n:] = math.nan
            for m in ("k", "v"):
                x[m][b, :, max(0, n + S - T):] = math.nan
    return x, d_out


def within(name, got, ref, bound, norm):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape and torch.equal(torch.isinf(got), torch.isinf(ref)), name
    fin = torch.isfinite(ref)
    err = (got - ref)[fin].abs()
    rel = (err.norm() / ref[fin].norm().clamp(min=1e-30)).item()
    worst = (err / bound[fin].clamp(min=1e-37)).max().item() if err.numel() else 0.0
    print("%-4s rel %.2e, of the bound %.2f" % (name, rel, worst), flush=True)
    assert not torch.isnan(got).any(), name
    assert (err <= bound[fin] + 1e-37).all(), (name, worst)
    # (a query that sees one key has P = 1 and dS = u - D = 0: what is left of such gradients
    # is rounding alone, held to the elements' bounds)
    if ref[fin].norm() > bound[fin].norm() and ref[fin].numel() >= 256:
        assert rel <= norm, (name, rel)


CASES = [  # B, HK, H, T, S, d, left, right
    (1, 1, 1, 1, 1, 8, -1, 0), (2, 1, 3, 1, 200, 64, -1, 0), (1, 2, 2, 5, 3, 16, -1, 0),
    (2, 2, 4, 33, 33, 64, 0, 0), (1, 1, 2, 129, 129, 128, 64, 0), (2, 1, 1, 100, 163, 40, 31, 0),
    (1, 2, 6, 260, 260, 72, -1, -1), (1, 1, 1, 150, 70, 32, 20, -1), (2, 2, 2, 65, 300, 96, 100, 7),
    (1, 1, 5, 257, 257, 24, 1 << 30, 1), (1, 3, 3, 192, 192, 128, -1, 0), (1, 1, 1, 300, 300, 64, 63, 0),
    (3, 1, 2, 64, 64, 120, 2147483647, 2147483647), (1, 1, 1, 40, 400, 16, 5, 0),
    # (few tiles of queries, or of keys, that see many: split into stretches and joined)
    (1, 1, 1, 130, 700, 64, -1, 0), (1, 1, 2, 64, 2000, 128, -1, -1), (1, 2, 8, 300, 300, 64, -1, 0),
    (2, 1, 4, 70, 900, 32, 600, 0), (1, 1, 1, 1, 1500, 72, -1, 0), (1, 1, 1, 900, 33, 40, -1, -1),
    # (key heads that 8 does not divide)
    (5, 2, 4, 140, 150, 64, 90, 0), (3, 3, 3, 260, 260, 128, -1, 0), (4, 4, 8, 40, 40, 32, 10, 3)]


@pytest.mark.parametrize("c", CASES)
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("ragged", [False, True])
def test_forward_backward(c, io, ragged):
    B, HK, H, T, S, d, left, right = c
    print("attention", c, io, ragged, flush=True)
    lengths = torch.tensor(([T - 1, 0, T + 5, T // 2, T] if T > 1 else [0, 1, -3])[:B]) if ragged else None
    check(B, HK, H, T, S, d, left, right, io, lengths)


def check(B, HK, H, T, S, d, left, right, io, lengths):
    """Forward and backward (ragged: other strides, and with a gradient of lse)."""
    ragged = lengths is not None
    layout = "bthd" if ragged else "bhtd"
    x, d_out = inputs(B, HK, H, T, S, d, io, d + T, lengths)
    d_lse = torch.randn(B, H, T, generator=torch.Generator().manual_seed(1)).double() if ragged else None
    sc = d ** -0.5
    out, lse, ref, a = attnref.gradients(x, sc, left, right, lengths, d_out, d_lse)
    bd = attnref.bounds(a, out, lse, sc, HK, io == "bf16")
    cfg = e2ttt.AttentionConfig(B, HK, H, T, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, S=S,
                                scale=sc, left=left, right=right)
    t = {n: dev(v, io, layout) for n, v in x.items()}
    tl = None if lengths is None else lengths.to(torch.int32).cuda()
    o, l = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"], lengths=tl)
    n1, n2 = (2.0 ** -8, 1.5 * 2.0 ** -8) if io == "bf16" else (2.0 ** -18, 2.0 ** -18)
    within("out", o, out, bd["out"], n1)
    within("lse", l, lse, bd["lse"], 2.0 ** -18)
    g = e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], o, l, dev(d_out, io, layout),
                                 None if d_lse is None else d_lse.float().cuda(), lengths=tl)
    for n, lim in (("q", n2), ("k", n2), ("v", n1)):
        within("d" + n, g["d" + n], ref[n], 1.01 * bd[n] + bd["own"] * ref[n].abs(), lim)


def make(B, HK, H, T, S, d, io="bf16", seed=0, **kw):
    x, d_out = inputs(B, HK, H, T, S, d, io, seed, size=kw.pop("size", 1.0))
    cfg = e2ttt.AttentionConfig(B, HK, H, T, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, S=S,
                                scale=kw.pop("scale", d ** -0.5), **kw)
    return cfg, {n: dev(v, io, "bhtd") for n, v in x.items()}, dev(d_out, io, "bhtd"), x, d_out


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_logits_far_apart(io):
    """Scores of some hundreds: all but a few probabilities vanish, the sum stays one."""
    cfg, t, tg, x, d_out = make(1, 1, 2, 140, 140, 64, io, size=6.0, scale=1.0)
    out, lse, ref, a = attnref.gradients(x, 1.0, -1, 0, None, d_out)
    bd = attnref.bounds(a, out, lse, 1.0, 1, io == "bf16")
    o, l = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"])
    within("out", o, out, bd["out"], math.inf)
    within("lse", l, lse, bd["lse"], 2.0 ** -18)
    g = e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], o, l, tg)
    for n in "qkv":
        within("d" + n, g["d" + n], ref[n], 1.01 * bd[n] + bd["own"] * ref[n].abs(), math.inf)


def test_keys_that_rise():
    """The running maximum grows with every tile of keys."""
    T, d = 400, 64
    x, d_out = inputs(1, 1, 1, T, T, d, "bf16", 5)
    x["k"] = rounded(x["q"].mean(2, keepdim=True) + torch.linspace(0, 30, T, dtype=torch.float64)[:, None] *
                     torch.ones(d, dtype=torch.float64) / d, "bf16")
    x["q"] = rounded(x["q"] * 0.1 + 1.0, "bf16")
    out, lse, a = attnref.attention(x, 1.0, -1, -1, None)
    cfg = e2ttt.AttentionConfig(1, 1, 1, T, d, scale=1.0, right=-1)
    o, l = e2ttt.attention_forward(cfg, *(dev(x[n], "bf16", "bhtd") for n in "qkv"))
    bd = attnref.bounds(a, out, lse, 1.0, 1, True)
    within("out", o, out, bd["out"], 2.0 ** -8)
    within("lse", l, lse, bd["lse"], 2.0 ** -18)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_autograd_of_shared_and_broadcast_inputs(io):
    """AttentionFunction: leaves used twice, keys that repeat over the batch, an
    upstream gradient without storage of its own, out alone and lse alone."""
    B, HK, H, T, d = 2, 2, 4, 70, 64
    x, _ = inputs(B, HK, H, T, T, d, io, 11)
    x["k"], x["v"] = x["k"][:1], x["v"][:1]
    cfg = e2ttt.AttentionConfig(B, HK, H, T, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32,
                                scale=0.125, left=40)
    t = {n: dev(v, io, "bhtd").requires_grad_(True) for n, v in x.items()}
    wide = {n: v.expand(B, -1, -1, -1) for n, v in x.items()}
    for which in ("out", "lse"):
        out, lse = e2ttt.AttentionFunction.apply(cfg, t["q"], t["k"].expand(B, -1, -1, -1),
                                                 t["v"].expand(B, -1, -1, -1))
        (out if which == "out" else lse).sum().backward()
        one = torch.ones(B, H, T, d, dtype=torch.float64)
        g0 = one if which == "out" else 0 * one
        o, l, ref, a = attnref.gradients(wide, 0.125, 40, 0, None, g0,
                                         None if which == "out" else one[..., 0])
        bd = attnref.bounds(a, o, l, 0.125, HK, io == "bf16")
        for n in "qkv":
            r, lim = ref[n], 1.01 * bd[n] + bd["own"] * ref[n].abs()
            if n != "q":        # (two gradients rounded, added and rounded)
                lim = lim.sum(0, keepdim=True) + (bd["own"] * r.abs()).sum(0, keepdim=True) * 1.02
                r = r.sum(0, keepdim=True)
            within("d" + n, t[n].grad, r, lim, math.inf)
            t[n].grad = None


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_strided_views(io):
    """q, k, v as slices of one projection [B, T, (H + 2 HK) d], gradients into such a tensor."""
    B, HK, H, T, d = 2, 2, 4, 90, 64
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(B, T, (H + 2 * HK) * d, generator=g).to(dt).cuda()
    cut = lambda t: (t[..., :H * d].unflatten(-1, (H, d)).transpose(1, 2),
                     t[..., H * d:(H + HK) * d].unflatten(-1, (HK, d)).transpose(1, 2),
                     t[..., (H + HK) * d:].unflatten(-1, (HK, d)).transpose(1, 2))
    cfg = e2ttt.AttentionConfig(B, HK, H, T, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32,
                                scale=0.125, left=33)
    q, k, v = cut(qkv)
    d_out = torch.randn(B, H, T, d, generator=g).to(dt).cuda()
    o1, l1 = e2ttt.attention_forward(cfg, q, k, v)
    o2, l2 = e2ttt.attention_forward(cfg, *(x.contiguous() for x in (q, k, v)))
    assert torch.equal(o1, o2) and torch.equal(l1, l2)
    into = torch.full_like(qkv, math.nan)
    dq, dk, dv = cut(into)
    e2ttt.attention_backward(cfg, q, k, v, o1, l1, d_out, grads=dict(dq=dq, dk=dk, dv=dv))
    ref = e2ttt.attention_backward(cfg, q.contiguous(), k.contiguous(), v.contiguous(), o2, l2, d_out)
    assert torch.equal(dq, ref["dq"]) and torch.equal(dk, ref["dk"]) and torch.equal(dv, ref["dv"])


def test_graph_and_other_stream():
    """Forward and backward captured once and replayed on new inputs, between eager calls
    on another stream: as the eager results, bit for bit."""
    cfg, t, tg, _, _ = make(2, 2, 4, 200, 200, 64, seed=1, left=70)
    out, lse = torch.empty_like(t["q"]), torch.empty(2, 4, 200, device="cuda")
    grads = {"d" + n: torch.empty_like(t[n]) for n in "qkv"}
    scratch = torch.empty(e2ttt.attention_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")

    def both():
        e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"], out=out, lse=lse)
        e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], out, lse, tg, grads=grads, scratch=scratch)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    other = torch.cuda.Stream()
    for i in range(4):
        _, t2, tg2, _, _ = make(2, 2, 4, 200, 200, 64, seed=20 + i, left=70)
        for n in "qkv":
            t[n].copy_(t2[n])
        tg.copy_(tg2)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            o, l = e2ttt.attention_forward(cfg, t2["q"], t2["k"], t2["v"])
            ref = e2ttt.attention_backward(cfg, t2["q"], t2["k"], t2["v"], o, l, tg2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, l)
        assert all(torch.equal(grads[n], ref[n]) for n in ref)


def test_lse_not_wanted_and_workspace_given():
    """The C entry without lse, and a split call on a workspace of the caller's."""
    import ctypes
    cfg, t, _, _, _ = make(1, 1, 2, 100, 1500, 64, seed=2)
    n = e2ttt.attention_workspace_bytes(cfg)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    o, l = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"], workspace=ws)
    o2 = torch.full_like(o, math.nan)
    p = lambda x: x.data_ptr()
    st = e2ttt.load().e2ttt_attn_forward(ctypes.byref(cfg.desc()), None, p(t["q"]), p(t["k"]), p(t["v"]),
                                         None, p(o2), None, p(ws), n, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(o, o2)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_smallest_and_largest_scale(io):
    """Scores that all vanish (a mean of the values) and the largest scale there is."""
    cfg, t, _, x, _ = make(1, 1, 1, 70, 70, 32, io, scale=2.0 ** -126)
    o, l = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"])
    n = torch.arange(1, 71, dtype=torch.float64)
    ref = x["v"].cumsum(2) / n[:, None]
    u = 2.0 ** -7 if io == "bf16" else 2.0 ** -17      # (a sum of 70 terms, its rounding, the out's)
    assert ((o.double().cpu() - ref).abs() <= u * x["v"].abs().cumsum(2) / n[:, None] + 1e-30).all()
    assert (l.double().cpu() - n.log()).abs().max() <= 2.0 ** -20
    k = dict(t, q=torch.zeros_like(t["q"]))
    cfg = e2ttt.AttentionConfig(1, 1, 1, 70, 32, cfg.io, scale=2.0 ** 127)
    o2, _ = e2ttt.attention_forward(cfg, k["q"], k["k"], k["v"])
    assert torch.equal(o2, o)


def test_split_calls_as_graphs_on_two_streams():
    """Two captured split calls with workspaces of their own, replayed at once."""
    runs = []
    for seed in (1, 2):
        cfg, t, tg, _, _ = make(1, 1, 4, 130, 1300, 64, seed=seed)
        o, l = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"])
        ref = e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], o, l, tg)
        ws = torch.empty(e2ttt.attention_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        sc = torch.empty(e2ttt.attention_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
        assert ws.numel() and sc.numel() > 8 * 4 * 130 * 2
        o2, l2, g2 = torch.empty_like(o), torch.empty_like(l), {n: torch.empty_like(x) for n, x in ref.items()}
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"], out=o2, lse=l2, workspace=ws)
            e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], o2, l2, tg, grads=g2, scratch=sc)
        runs.append((graph, torch.cuda.Stream(), o, l, ref, o2, l2, g2, ws, sc, t, tg))
    for _ in range(4):
        for r in runs:
            for x in (r[5], r[6], *r[7].values()):
                x.zero_()
        torch.cuda.synchronize()
        for r in runs:
            with torch.cuda.stream(r[1]):
                r[0].replay()
        torch.cuda.synchronize()
        for _, _, o, l, ref, o2, l2, g2, *_ in runs:
            assert torch.equal(o, o2) and torch.equal(l, l2)
            assert all(torch.equal(ref[n], g2[n]) for n in ref)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,T,S,d,n,left", [
    (1, 2, 40, 40, 64, 5, -1), (2, 2, 150, 150, 128, 40, 20),   # live rows, then dead ones in their tile
    (1, 1, 40, 10, 32, 40, -1),                                 # queries ahead of the first key
    (1, 1, 16, 4096, 64, 7, -1), (1, 1, 40, 4096, 128, 9, -1)])  # split
def test_zeros_beside_infinities(B, H, T, S, d, n, left, io):
    """What is not live, and what sees nothing, is zero also where live values of its
    tile are infinite."""
    cfg, x, g, _, _ = make(B, 1, H, T, S, d, io, left=left)
    q, k, v = x["q"], x["k"], x["v"]
    lengths = torch.full((B,), n, dtype=torch.int32, device="cuda")
    end = n + S - T
    first = max(0, T - S)             # of the queries with a key
    k[:, :, end - 2] = math.inf
    v[:, :, end - 1] = math.inf
    out, lse = e2ttt.attention_forward(cfg, q, k, v, lengths=lengths)
    dead = torch.ones(T, dtype=torch.bool, device=q.device)
    dead[first:n] = False
    assert (out[:, :, dead] == 0).all() and (lse[:, :, dead] == -math.inf).all()
    assert not torch.isfinite(out[:, :, n - 1]).any()
    g[:, :, n - 1] = math.inf
    r = e2ttt.attention_backward(cfg, q, k, v, out, lse, g, lengths=lengths)
    assert (r["dq"][:, :, dead] == 0).all()
    assert (r["dk"][:, :, end:] == 0).all() and (r["dv"][:, :, end:] == 0).all()


@pytest.mark.parametrize("io,B,HK,H,T,S,d,left,right,ragged", [
    ("bf16", 1, 9, 9, 2570, 2570, 64, -1, 0, True),      # in two, both directions
    ("f32", 1, 32, 32, 700, 700, 16, -1, 0, False),
    ("bf16", 9, 1, 3, 900, 900, 64, -1, 3, True),        # heads dealt in threes; one of nine behind
    ("bf16", 8, 1, 2, 700, 700, 32, 2, -1, False),       # long rows the other way round
    ("bf16", 16, 1, 1, 300, 290, 128, -1, 0, True),      # in pairs
    ("bf16", 15, 8, 8, 600, 600, 128, -1, 0, True),      # thirteen and two; twice seven and one
    ("f32", 4, 2, 6, 600, 600, 72, -1, 0, True)])
def test_rows_of_unequal_length(io, B, HK, H, T, S, d, left, right, ragged):
    """Each workgroup's place in its launch, and the stretches that are joined."""
    lengths = torch.randint(T // 3, T + 1, (B,), generator=torch.Generator().manual_seed(T)) if ragged else None
    check(B, HK, H, T, S, d, left, right, io, lengths)


def test_first_rows_of_split_calls():
    """Rows that see few keys take the same D, and so the same dS, whether their call is
    split (189 tiles) or not (378): sums in another order alone, some 2^-20, which turn
    a rounding of 2^-8 in 2^-11 of all elements, 2^-13 in the 2-norm.  D from a bf16 out
    alone would leave about 2^-8."""
    cfg, x, g, _, _ = make(2, 9, 9, 2570, 2570, 64, seed=3)
    one = dataclasses.replace(cfg, B=1)
    got = []
    for c, n in ((cfg, 2), (one, 1)):
        q, k, v = (x[m][:n] for m in "qkv")
        out, lse = e2ttt.attention_forward(c, q, k, v)
        got.append(e2ttt.attention_backward(c, q, k, v, out, lse, g[:n])["dq"][0, :, :128].float())
    a, b = got
    assert (a - b).norm() <= 2.0 ** -12 * a.norm()


RANGE = [  # T, S, d (the last two are split)
    (70, 70, 32), (40, 30, 64), (130, 130, 128), (16, 4096, 64), (20, 4000, 128)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("c", RANGE)
@pytest.mark.parametrize("how", ["up", "down", "raw"])
def test_scores_out_of_range(c, how, io):
    """Finite queries and keys whose scores pass the range of fp32, as q . k or times the
    scale: NaN, in the gradients of the queries too, and not the zeros of a query that
    sees no key; those keep theirs."""
    T, S, d = c
    cfg, t, tg, _, _ = make(2, 1, 2, T, S, d, io, scale=2.0 ** 127 if how != "raw" else 1.0)
    q, k = t["q"].fill_(1.0 if how != "raw" else 1e25), t["k"].fill_(1.0)
    if how != "up":
        k.fill_(-1.0 if how == "down" else -1e25)
    lengths = torch.tensor([T, T - 3], dtype=torch.int32, device="cuda")
    out, lse = e2ttt.attention_forward(cfg, q, k, t["v"], lengths=lengths)
    sees = torch.zeros(2, T, dtype=torch.bool, device="cuda")
    sees[0, max(0, T - S):] = sees[1, max(0, T - S):T - 3] = True
    sees = sees[:, None].expand(2, 2, T)
    assert torch.isnan(out[sees]).all() and torch.isnan(lse[sees]).all()
    assert (out[~sees] == 0).all() and (lse[~sees] == -math.inf).all()
    g = e2ttt.attention_backward(cfg, q, k, t["v"], out, lse, tg, lengths=lengths)
    assert torch.isnan(g["dq"][sees]).all() and (g["dq"][~sees] == 0).all()
    end = T - 3 + S - T
    assert (g["dk"][1, :, end:] == 0).all() and (g["dv"][1, :, end:] == 0).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("S", [200, 4096])
def test_keys_whose_scores_vanish_below_the_range(S, io):
    """A whole stretch of keys with q . k below fp32's range weighs nothing beside
    the other keys: as the same call without them."""
    d, T, n = 64, 16, S // 2
    cfg, t, _, x, _ = make(1, 1, 2, T, S, d, io, right=-1, scale=1.0)
    q = torch.full_like(t["q"], 1e25)
    q[..., 1:] = 0.0
    k = torch.zeros_like(t["k"])
    k[:, :, :n, 0] = -1e25
    out, lse = e2ttt.attention_forward(cfg, q, k, t["v"])
    ref = x["v"][:, :, n:].mean(2, keepdim=True).expand(1, 2, T, d)
    # (sums of S terms, their rounding to the type and, bf16, one of the weights, here exact)
    u = attnref.UBF if io == "bf16" else 0.0
    lim = attnref.U32 * (S + 8) * x["v"][:, :, n:].abs().mean(2, keepdim=True) + u * ref.abs()
    assert ((out.double().cpu() - ref).abs() <= 1.01 * lim).all()
    assert (lse.double().cpu() - math.log(S - n)).abs().max() <= 2.0 ** -20


def test_an_lse_that_leaves_the_range():
    """An lse that fp32 holds but not times log2 e: no gradient of zero."""
    cfg, t, tg, _, _ = make(1, 1, 1, 40, 40, 32)
    out, lse = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"])
    lse[0, 0, 7] = 3e38
    g = e2ttt.attention_backward(cfg, t["q"], t["k"], t["v"], out, lse, tg)
    assert torch.isnan(g["dq"][0, 0, 7]).all() and torch.isfinite(g["dq"][0, 0, :7]).all()


def test_autograd_in_a_capture():
    """A capture that wants gradients is refused and can go on; without them the call is
    captured as any other."""
    cfg, t, tg, _, _ = make(1, 1, 2, 70, 70, 64)
    leaves = [t[n].detach().clone().requires_grad_(True) for n in "qkv"]
    ref, _ = e2ttt.attention_forward(cfg, t["q"], t["k"], t["v"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="attention_forward and attention_backward"):
            e2ttt.AttentionFunction.apply(cfg, *leaves)
        with torch.no_grad():
            out, _ = e2ttt.AttentionFunction.apply(cfg, *leaves)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        got, _ = e2ttt.AttentionFunction.apply(cfg, *leaves)
        assert torch.equal(got.detach(), ref)
    assert all(torch.isfinite(g).all() for g in torch.autograd.grad(got, leaves, tg))


@pytest.mark.parametrize("io,B,HK,H,T,S,d,ragged", [
    ("bf16", 1, 65, 1040, 160, 160, 72, True),     # dk and dv, 130 groups
    ("f32", 1, 26, 26, 700, 700, 16, False)])      # 156, both directions
def test_rows_of_unequal_length_on_half_of_the_card(io, B, HK, H, T, S, d, ragged):
    """129 to 160 groups are split in two as those on either side of them are."""
    cfg = e2ttt.AttentionConfig(B, HK, H, T, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, S=S)
    rows, part = -(-4 * B * H * T // 256) * 256, 8 * B * HK * S * d
    assert e2ttt.attention_scratch_bytes(cfg) == 2 * rows + 2 * part
    lengths = torch.randint(T // 3, T + 1, (B,), generator=torch.Generator().manual_seed(T)) if ragged else None
    check(B, HK, H, T, S, d, -1, 0, io, lengths)
