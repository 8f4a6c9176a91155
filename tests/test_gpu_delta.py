"""GPU parity of the gated delta rule (forward, backward, recurrent form) with
the token-by-token recurrence in 64 bits (tests/deltaref.py).

Tolerances, set before any run of these kernels.  A bf16 output is rounded
once, at most 2^-8 of its value.  Everything else is fp32: a value passes at
most 16 roundings of 2^-24 on its way (state, K W, R, T, U, P, decayed U and
their adjoints, over the few chunks within which the decaying state forgets),
each a sum over up to 256 terms whose roundings grow as the root, 16: in the
worst case 2^-16 in the 2-norm; 2^-18 is asked for, and 2^-8 + 2^-14 of bf16
outputs (products that only reach those drop terms below 2^-17).
"""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import deltaref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def make(B, HK, H, T, dk, dv, io, seed=0, decay=True, state=True, rate=1.0):
    """Inputs on the CPU in float64, already rounded to their types."""
    g = torch.Generator().manual_seed(1000 * seed + 17 * T + dk + dv)
    dt = torch.bfloat16 if io == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    def unit(x):
        return (x / x.norm(dim=-1, keepdim=True)).to(dt).double()

    x = dict(q=unit(rn(B, HK, T, dk)), k=unit(rn(B, HK, T, dk)), v=rn(B, H, T, dv).to(dt).double(),
             eta=torch.sigmoid(rn(B, H, T)).float().double())
    x["log_gamma"] = (-rate * torch.nn.functional.softplus(rn(B, H, T) - 2)).float().double() if decay else None
    x["w_in"] = (0.3 * rn(B, H, dv, dk)).float().double() if state else None
    d = dict(d_out=rn(B, H, T, dv).to(dt).double(), d_w_out=(0.3 * rn(B, H, dv, dk)).float().double())
    return x, d


def dev(t, io, layout="bhtd"):
    """To the GPU in its type; token tensors of layout bthd as views of that order."""
    if t is None:
        return None
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    t = t.to(dt).cuda()
    return t.transpose(1, 2).contiguous().transpose(1, 2) if layout == "bthd" else t


def to_dev(x, io, layout="bhtd"):
    return {n: dev(t, io if n in ("q", "k", "v", "d_out") else "f32",
                   layout if n not in ("w_in", "d_w_out") else "bhtd") for n, t in x.items()}


def close(name, got, ref, io_type):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), name
    tol = (2.0 ** -8 + 2.0 ** -14) if io_type == "bf16" else 2.0 ** -18
    n = ref.norm().item()
    err = (got - ref).norm().item()
    print("%-12s rel %.2e" % (name, err / max(n, 1e-30)), flush=True)
    assert err <= tol * n + 1e-30, (name, err / max(n, 1e-30), tol)


def check(x, d, c, io, layout="bhtd", lengths=None, use_d_w=True, tag=""):
    B, HK, H, T, dk, dv = c
    scale = dk ** -0.5
    cfg = e2ttt.DeltaConfig(B, HK, H, T, dk, dv, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, scale)
    print("delta", c, io, layout, tag, flush=True)
    t, td = to_dev(x, io, layout), to_dev(d, io, layout)
    ln = None if lengths is None else torch.as_tensor(lengths).to(torch.int32)
    lg = None if ln is None else ln.cuda()
    out, w_out, ws = e2ttt.delta_forward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"],
                                         t["w_in"], lengths=lg, save_for_backward=True)
    g = e2ttt.delta_backward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], ws, td["d_out"],
                             td["d_w_out"] if use_d_w else None, lengths=lg)
    out2, w_out2, _ = e2ttt.delta_forward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"],
                                          t["w_in"], lengths=lg)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(w_out, w_out2)     # saving changes nothing
    ro, rw, rg = deltaref.delta_grads(x, scale, d["d_out"], d["d_w_out"] if use_d_w else None, ln)
    close("out", out, ro, io)
    close("w_out", w_out, rw, "f32")
    for n, m in (("q", "dq"), ("k", "dk"), ("v", "dv")):
        close(m, g[m], rg[n], io)
    close("d_eta", g["d_eta"], rg["eta"], "f32")
    if x["log_gamma"] is not None:
        close("d_log_gamma", g["d_log_gamma"], rg["log_gamma"], "f32")
    if x["w_in"] is not None:
        close("d_w_in", g["d_w_in"], rg["w_in"], "f32")
    return out, g


SIZES = [(1, 1, 1, 1, 16, 16), (1, 1, 1, 2, 8, 8), (2, 1, 2, 63, 64, 64), (1, 2, 2, 64, 64, 64),
         (1, 1, 3, 65, 32, 24), (2, 2, 4, 130, 64, 120), (1, 1, 1, 200, 128, 128),
         (1, 1, 2, 97, 72, 256), (3, 1, 1, 129, 128, 40)]


@pytest.mark.parametrize("c", SIZES)
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_sizes(c, io):
    x, d = make(*c, io)
    check(x, d, c, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
@pytest.mark.parametrize("decay,state", [(True, False), (False, True), (False, False)])
def test_options(io, layout, decay, state):
    c = (2, 2, 4, 100, 64, 72)
    x, d = make(*c, io, decay=decay, state=state, seed=3)
    check(x, d, c, io, layout, use_d_w=state)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [(0, 1, 150, 64), (150, 0, 0, 65), (-5, 1000, 128, 149)])
def test_lengths(io, lengths):
    # padded rows hold NaN: they are not read, and come back as zero
    c = (4, 1, 2, 150, 64, 64)
    x, d = make(*c, io, seed=5)
    y, e = dict(x), dict(d)
    for n in ("q", "k", "v", "eta", "log_gamma"):
        y[n] = x[n].clone()
        for b, l in enumerate(lengths):
            y[n][b, :, max(0, l):] = float("nan")
    e["d_out"] = d["d_out"].clone()
    for b, l in enumerate(lengths):
        e["d_out"][b, :, max(0, l):] = float("nan")
    z = {n: t.clone() if t is not None else None for n, t in x.items()}
    dd = dict(d, d_out=torch.nan_to_num(e["d_out"]))
    scale = c[4] ** -0.5
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, scale)
    t, td = to_dev(y, io), to_dev(e, io)
    lg = torch.tensor(lengths, dtype=torch.int32).cuda()
    out, w_out, ws = e2ttt.delta_forward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"],
                                         t["w_in"], lengths=lg, save_for_backward=True)
    g = e2ttt.delta_backward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], ws, td["d_out"],
                             td["d_w_out"], lengths=lg)
    torch.cuda.synchronize()
    ln = torch.tensor(lengths).clamp(0, c[3])
    ro, rw, rg = deltaref.delta_grads(z, scale, dd["d_out"], dd["d_w_out"], ln)
    for n, got, ref, ty in (("out", out, ro, io), ("w_out", w_out, rw, "f32"), ("dq", g["dq"], rg["q"], io),
                            ("dk", g["dk"], rg["k"], io), ("dv", g["dv"], rg["v"], io),
                            ("d_eta", g["d_eta"], rg["eta"], "f32"),
                            ("d_log_gamma", g["d_log_gamma"], rg["log_gamma"], "f32"),
                            ("d_w_in", g["d_w_in"], rg["w_in"], "f32")):
        close(n, got, ref, ty)
    for b, l in enumerate(ln.tolist()):
        for got in (out, g["dq"], g["dk"], g["dv"], g["d_eta"], g["d_log_gamma"]):
            assert (got[b, :, l:] == 0).all()
        if l == 0:
            assert torch.equal(w_out[b], t["w_in"][b])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_gates_at_their_ends(io):
    """eta 0 and 1, decays of nothing, of 1e-20 and to nothing (-inf), next to each other."""
    c = (1, 1, 2, 140, 64, 64)
    x, d = make(*c, io, seed=7)
    x["eta"][:, 0, ::3] = 0.0
    x["eta"][:, 0, 1::3] = 1.0
    x["eta"][:, 1, 5] = 1e-30
    x["eta"][:, 1, 70:80] = 0.0
    x["log_gamma"][:, 0, ::7] = 0.0
    x["log_gamma"][:, 0, 40] = -float("inf")
    x["log_gamma"][:, 0, 64:67] = -float("inf")
    x["log_gamma"][:, 1, 100:120] = -46.0
    # (the reference's gradient at -inf is 0 * inf; the clamped value has the same exp)
    y = dict(x, log_gamma=x["log_gamma"].clamp(min=-800.0))
    scale = c[4] ** -0.5
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, scale)
    t, td = to_dev(x, io), to_dev(d, io)
    out, w_out, ws = e2ttt.delta_forward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"],
                                         t["w_in"], save_for_backward=True)
    g = e2ttt.delta_backward(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], ws, td["d_out"],
                             td["d_w_out"])
    ro, rw, rg = deltaref.delta_grads(y, scale, d["d_out"], d["d_w_out"])
    for n, got, ref, ty in (("out", out, ro, io), ("w_out", w_out, rw, "f32"), ("dq", g["dq"], rg["q"], io),
                            ("dk", g["dk"], rg["k"], io), ("dv", g["dv"], rg["v"], io),
                            ("d_eta", g["d_eta"], rg["eta"], "f32"),
                            ("d_log_gamma", g["d_log_gamma"], rg["log_gamma"], "f32"),
                            ("d_w_in", g["d_w_in"], rg["w_in"], "f32")):
        close(n, got, ref, ty)


@pytest.mark.parametrize("c", [(1, 1, 1, 1, 16, 16), (3, 2, 4, 1, 64, 64), (2, 1, 2, 5, 128, 128),
                               (2, 1, 3, 3, 72, 200), (2, 2, 2, 2, 24, 8)])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_step(c, io, layout):
    B, HK, H, T, dk, dv = c
    x, _ = make(*c, io, seed=11)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 0.5)
    t = to_dev(x, io, layout)
    ro, rw = deltaref.delta(x["q"], x["k"], x["v"], x["eta"], x["log_gamma"], x["w_in"], 0.5)
    w = t["w_in"].clone()
    out = e2ttt.delta_step(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], w)
    close("out", out, ro, io)
    close("w", w, rw, "f32")
    # a pool: the sequences in other slots, the rest untouched
    pool = torch.randn(2 * B + 1, H, dv, dk, device="cuda")
    slots = torch.arange(2 * B - 1, -1, -2, dtype=torch.int32, device="cuda")[:B].contiguous()
    before = pool.clone()
    pool[slots.long()] = t["w_in"]
    out2 = e2ttt.delta_step(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], pool, slots=slots)
    assert torch.equal(out2, out) and torch.equal(pool[slots.long()], w)
    rest = [i for i in range(2 * B + 1) if i not in slots.tolist()]
    assert torch.equal(pool[rest], before[rest])


def test_step_slots_skipped_and_shared():
    c = (70, 1, 2, 2, 64, 64)
    x, _ = make(*c, "f32", seed=13)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_F32, 1.0)
    t = to_dev(x, "f32")
    slots = [(7 * b) % 30 for b in range(70)]
    slots[3] = -1
    slots[69] = 30              # one past the pool
    slots[5] = slots[68] = 4    # among others at the same slot
    pool = t["w_in"][:30].clone()
    out = e2ttt.delta_step(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], pool,
                           slots=torch.tensor(slots, dtype=torch.int32).cuda())
    w = x["w_in"][:30].clone()
    ref = torch.zeros(70, 2, 2, 64, dtype=torch.float64)
    for b, s in enumerate(slots):
        if 0 <= s < 30:
            a = [x[n][b:b + 1] for n in ("q", "k", "v", "eta", "log_gamma")]
            ref[b:b + 1], w[s:s + 1] = deltaref.delta(*a, w[s:s + 1], 1.0)
    close("out", out, ref, "f32")
    close("w", pool, w, "f32")
    assert (out[3] == 0).all() and (out[69] == 0).all()


def test_autograd_and_differences():
    """DeltaFunction's gradients against central differences of the 64-bit rule."""
    c = (1, 1, 2, 70, 16, 16)
    x, d = make(*c, "f32", seed=17)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_F32, 1.0)
    t = {n: a.requires_grad_(True) for n, a in to_dev(x, "f32").items()}
    out, w_out = e2ttt.DeltaFunction.apply(cfg, t["q"], t["k"], t["v"], t["eta"], t["log_gamma"], t["w_in"])
    loss = (out * d["d_out"].float().cuda()).sum() + (w_out * d["d_w_out"].float().cuda()).sum()
    grads = torch.autograd.grad(loss, list(t.values()))

    def f(y):
        o, w = deltaref.delta(y["q"], y["k"], y["v"], y["eta"], y["log_gamma"], y["w_in"], 1.0)
        return ((o * d["d_out"]).sum() + (w * d["d_w_out"]).sum()).item()

    gen = torch.Generator().manual_seed(1)
    for n, gr in zip(t, grads):
        u = torch.randn(x[n].shape, generator=gen, dtype=torch.float64)
        h = 1e-5
        num = (f(dict(x, **{n: x[n] + h * u})) - f(dict(x, **{n: x[n] - h * u}))) / (2 * h)
        got = (gr.double().cpu() * u).sum().item()
        # h^2 of third derivatives, and the fp32 gradient's 2^-18 in the 2-norm times |u|
        tol = 1e-6 * abs(num) + 2.0 ** -18 * gr.double().norm().item() * u.norm().item()
        assert abs(got - num) <= tol, (n, got, num)


def test_only_one_output_used():
    c = (1, 1, 1, 66, 32, 32)
    x, d = make(*c, "f32", seed=19)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_F32, 1.0)
    t = {n: a.requires_grad_(True) for n, a in to_dev(x, "f32").items()}
    _, w_out = e2ttt.DeltaFunction.apply(cfg, *[t[n] for n in ("q", "k", "v", "eta", "log_gamma", "w_in")])
    dq, dk = torch.autograd.grad((w_out * d["d_w_out"].float().cuda()).sum(), [t["q"], t["k"]])
    _, _, rg = deltaref.delta_grads(x, 1.0, torch.zeros_like(d["d_out"]), d["d_w_out"])
    assert (dq == 0).all()
    close("dk", dk, rg["k"], "f32")


def test_prefill_then_steps_equal_one_prefill():
    """A prompt, then decode token by token, against the whole sequence at once."""
    B, HK, H, T, n, dk, dv = 2, 1, 2, 90, 6, 64, 64
    x, _ = make(B, HK, H, T + n, dk, dv, "bf16", seed=23)
    t = to_dev(x, "bf16")
    io = e2ttt.DT_BF16
    whole = e2ttt.DeltaConfig(B, HK, H, T + n, dk, dv, io, 0.125)
    names = ("q", "k", "v", "eta", "log_gamma")
    out, w_out, _ = e2ttt.delta_forward(whole, *[t[m] for m in names], t["w_in"])
    pre = e2ttt.DeltaConfig(B, HK, H, T, dk, dv, io, 0.125)
    # views of the longer tensors: rows of the same strides
    o1, w, _ = e2ttt.delta_forward(pre, *[t[m][:, :, :T] for m in names], t["w_in"])
    one = e2ttt.DeltaConfig(B, HK, H, 1, dk, dv, io, 0.125)
    steps = [e2ttt.delta_step(one, *[t[m][:, :, T + i:T + i + 1] for m in names], w) for i in range(n)]
    close("out", torch.cat([o1] + steps, 2), out.double().cpu(), "bf16")
    close("w", w, w_out.double().cpu(), "f32")


def test_state_in_place_and_in_stretches():
    """w_out may be w_in, and a call of so many units that its chunks are taken in stretches
    carries its state over several launches: equal, bit for bit, to the calls of its parts;
    and saving for the backward in stretches gives what it gives in one."""
    B, HK, H, dk, dv = 64, 8, 32, 16, 16
    T = 64 * 5
    io = e2ttt.DT_BF16
    cfg = e2ttt.DeltaConfig(B, HK, H, T, dk, dv, io, 1.0)
    one_chunk = e2ttt.delta_workspace_bytes(e2ttt.DeltaConfig(B, HK, H, 64, dk, dv), False)
    assert e2ttt.delta_workspace_bytes(cfg, False) < 4 * one_chunk        # several stretches
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).bfloat16()
    q, k, v = unit(rn(B, HK, T, dk)), unit(rn(B, HK, T, dk)), rn(B, H, T, dv).bfloat16()
    eta, lg, w = torch.sigmoid(rn(B, H, T)), -torch.rand(B, H, T, device="cuda", generator=g), rn(B, H, dv, dk)
    out, w_out, _ = e2ttt.delta_forward(cfg, q, k, v, eta, lg, w)
    w2 = w.clone()
    parts = []
    for sl in (slice(0, 128), slice(128, T)):
        n = sl.stop - sl.start
        cfg2 = e2ttt.DeltaConfig(B, HK, H, n, dk, dv, io, 1.0)
        o, _, _ = e2ttt.delta_forward(cfg2, *[a[:, :, sl] for a in (q, k, v, eta, lg)], w2, w_out=w2)
        parts.append(o)
    assert torch.equal(torch.cat(parts, 2), out) and torch.equal(w2, w_out)
    o2, w3, ws = e2ttt.delta_forward(cfg, q, k, v, eta, lg, w, save_for_backward=True)
    assert torch.equal(o2, out) and torch.equal(w3, w_out)
    d_out = rn(B, H, T, dv).bfloat16()
    gr = e2ttt.delta_backward(cfg, q, k, v, eta, lg, ws, d_out)
    # the first sequence alone (a call of few units, in segments), to fp32 and bf16 rounding
    few = e2ttt.DeltaConfig(1, HK, H, T, dk, dv, io, 1.0)
    one = [a[:1].contiguous() for a in (q, k, v, eta, lg)]
    _, _, ws1 = e2ttt.delta_forward(few, *one, w[:1].contiguous(), save_for_backward=True)
    g1 = e2ttt.delta_backward(few, *one, ws1, d_out[:1].contiguous())
    for n, io_n in (("dq", "bf16"), ("dk", "bf16"), ("dv", "bf16"), ("d_eta", "f32"),
                    ("d_log_gamma", "f32"), ("d_w_in", "f32")):
        close(n, gr[n][:1], g1[n].double().cpu(), io_n)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("c,lengths", [((1, 1, 1, 1500, 64, 64), None), ((2, 1, 2, 1030, 128, 72), (1030, 700)),
                                       ((1, 2, 2, 801, 16, 40), None), ((2, 1, 1, 900, 72, 128), (0, 64))])
def test_segments(c, lengths, io):
    """Long chains of few units, which run as segments: forward and backward against the
    recurrence, and a decay slow enough that the first segment's state reaches the last."""
    x, d = make(*c, io, seed=31, rate=0.003)
    check(x, d, c, io, "bthd" if c[0] == 1 else "bhtd",
          lengths=None if lengths is None else torch.tensor(lengths))


def test_segments_in_place_and_in_stretches():
    """w_out = w_in where the call runs in segments, and a sequence of several stretches, each
    in segments, that carries its state from one to the next: bit for bit the separate calls."""
    c = (1, 1, 2, 2000, 64, 64)
    x, _ = make(*c, "bf16", seed=37, rate=0.01)
    t = to_dev(x, "bf16")
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 1.0)
    names = ("q", "k", "v", "eta", "log_gamma")
    out, w_out, _ = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"])
    for _ in range(8):
        w = t["w_in"].clone()
        o, _, _ = e2ttt.delta_forward(cfg, *[t[n] for n in names], w, w_out=w)
        assert torch.equal(o, out) and torch.equal(w, w_out)
    B, H, T, d = 1, 16, 64 * 1100, 64         # more fragments than a stretch holds
    cfg = e2ttt.DeltaConfig(B, H, H, T, d, d, e2ttt.DT_BF16, 1.0)
    each = e2ttt.delta_workspace_bytes(e2ttt.DeltaConfig(B, H, H, 64, d, d), False)
    assert e2ttt.delta_workspace_bytes(cfg, False) < 900 * each
    g = torch.Generator(device="cuda").manual_seed(3)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).bfloat16()
    a = [unit(rn(B, H, T, d)), unit(rn(B, H, T, d)), rn(B, H, T, d).bfloat16(),
         torch.sigmoid(rn(B, H, T)), -0.001 * torch.rand(B, H, T, device="cuda", generator=g)]
    w = rn(B, H, d, d)
    out, w_out, _ = e2ttt.delta_forward(cfg, *a, w)
    n = 64 * 550
    half = e2ttt.DeltaConfig(B, H, H, n, d, d, e2ttt.DT_BF16, 1.0)
    o1, w1, _ = e2ttt.delta_forward(half, *[y[:, :, :n] for y in a], w)
    o2, w2, _ = e2ttt.delta_forward(half, *[y[:, :, n:] for y in a], w1)
    assert torch.equal(torch.cat([o1, o2], 2), out) and torch.equal(w2, w_out)


def test_no_second_derivatives():
    c = (1, 1, 1, 10, 16, 16)
    x, _ = make(*c, "f32", seed=41)
    t = {n: a.requires_grad_(True) for n, a in to_dev(x, "f32").items()}
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_F32, 1.0)
    out, _ = e2ttt.DeltaFunction.apply(cfg, *[t[n] for n in ("q", "k", "v", "eta", "log_gamma", "w_in")])
    (dq,) = torch.autograd.grad(out.sum(), t["q"], create_graph=True)
    with pytest.raises(RuntimeError):
        dq.sum().backward()


def test_graph_replays_and_streams():
    """A training step captured as a graph and replayed equals the eager one, with eager work
    between the replays; and the calls on another stream equal those on the default one."""
    c = (2, 1, 2, 130, 64, 64)
    x, d = make(*c, "bf16", seed=29)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 0.125)
    t, td = to_dev(x, "bf16"), to_dev(d, "bf16")
    names = ("q", "k", "v", "eta", "log_gamma")
    ws = e2ttt.alloc_delta_workspace(cfg, True)
    sc = torch.empty(e2ttt.delta_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    out, w_out = torch.empty_like(t["v"]), torch.empty_like(t["w_in"])
    grads = dict(dq=torch.empty_like(t["q"]), dk=torch.empty_like(t["k"]), dv=torch.empty_like(t["v"]),
                 d_eta=torch.empty_like(t["eta"]), d_log_gamma=torch.empty_like(t["eta"]),
                 d_w_in=torch.empty_like(t["w_in"]))

    def step():
        e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"], out=out, w_out=w_out, workspace=ws,
                            save_for_backward=True)
        e2ttt.delta_backward(cfg, *[t[n] for n in names], ws, td["d_out"], td["d_w_out"], grads=grads,
                             scratch=sc)

    everything = lambda: [a.clone() for a in (out, w_out, *grads.values())]
    step()
    torch.cuda.synchronize()
    ref = everything()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(everything(), ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for a in (out, w_out, *grads.values()):
            a.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(everything(), ref)), i
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(everything(), ref)), i


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("c,lengths", [((3, 1, 2, 200, 64, 64), (70, 0, 130)),
                                       ((2, 1, 1, 1500, 32, 40), (600, 0))])
def test_nothing_behind_a_sequence(c, lengths, io):
    """Tokens behind a sequence's end have zero outputs and gradients whatever its live tokens
    and its state hold, and an empty sequence keeps its state as it is."""
    x, d = make(*c, io, seed=53)
    x["v"][0, :, 3, 5] = float("nan")
    x["k"][0, :, 40, 2] = float("inf")
    x["w_in"][1, 0, 1, 2] = float("inf")
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 0.125)
    t, td = to_dev(x, io), to_dev(d, io)
    names = ("q", "k", "v", "eta", "log_gamma")
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for save in (True, False):
        out = torch.full_like(t["v"], float("nan"))
        _, w_out, ws = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"], lengths=ln, out=out,
                                           save_for_backward=save)
        for b, n in enumerate(lengths):
            assert (out[b, :, n:] == 0).all(), (save, b)
        assert torch.equal(w_out[1], t["w_in"][1])
        if not save:
            continue
        g = {n: torch.full_like(a, float("nan")) for n, a in
             (("dq", t["q"]), ("dk", t["k"]), ("dv", t["v"]), ("d_eta", t["eta"]),
              ("d_log_gamma", t["eta"]), ("d_w_in", t["w_in"]))}
        e2ttt.delta_backward(cfg, *[t[n] for n in names], ws, td["d_out"], td["d_w_out"], lengths=ln,
                             grads=g)
        for n, a in g.items():
            for b, k in enumerate(lengths):
                if n != "d_w_in":
                    assert (a[b, :, k:] == 0).all(), (n, b)
        assert torch.equal(g["d_w_in"][1], td["d_w_out"][1])
    if len(lengths) == 3:          # the sequences with finite values are as they would be alone
        x["v"][0] = 0
        x["k"][0] = 0
        ref, rw, _ = deltaref.delta_grads({n: a[2:] for n, a in x.items()}, 0.125, d["d_out"][2:],
                                          d["d_w_out"][2:], torch.tensor(lengths[2:]))
        close("out", out[2:], ref, io)
        close("w_out", w_out[2:], rw, "f32")


@pytest.mark.parametrize("c,lengths", [((7, 4, 12, 2100, 40, 24), (2100, 0, 1, 700, 1024, 1025, 2099)),
                                       ((6, 16, 16, 2049, 64, 8), None)])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_parts(c, lengths, layout):
    """Units that half fill the card, over long sequences: the chain in parts."""
    x, d = make(*c, "bf16", seed=61)
    B, HK, H, T, dk, dv = c
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 0.125)
    t, td = to_dev(x, "bf16", layout), to_dev(d, "bf16", layout)
    names = ("q", "k", "v", "eta", "log_gamma")
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    lg = None if ln is None else ln.cuda()
    out, w_out, ws = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"], lengths=lg,
                                         save_for_backward=True)
    g = e2ttt.delta_backward(cfg, *[t[n] for n in names], ws, td["d_out"], td["d_w_out"], lengths=lg)
    w = t["w_in"].clone()
    out2, _, _ = e2ttt.delta_forward(cfg, *[t[n] for n in names], w, lengths=lg, w_out=w)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(w_out, w)
    for b in (0, 3, 5):            # (the sequences do not meet)
        ro, rw, rg = deltaref.delta_grads({n: a[b:b + 1] for n, a in x.items()}, 0.125, d["d_out"][b:b + 1],
                                          d["d_w_out"][b:b + 1], None if ln is None else ln[b:b + 1])
        close("out", out[b:b + 1], ro, "bf16")
        close("w_out", w_out[b:b + 1], rw, "f32")
        for n, m, y in (("q", "dq", "bf16"), ("k", "dk", "bf16"), ("v", "dv", "bf16"),
                        ("eta", "d_eta", "f32"), ("log_gamma", "d_log_gamma", "f32"),
                        ("w_in", "d_w_in", "f32")):
            close(m, g[m][b:b + 1], rg[n], y)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_far_tokens(io):
    """Tokens as far apart as they may be (2^23 elements, a chunk's offsets near 31 bits, a
    sequence's beyond 32) give what contiguous ones give, to the bit."""
    c, far = (1, 1, 1, 130, 64, 64), 1 << 23
    x, d = make(*c, io, seed=71)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 0.125)
    t, td = to_dev(x, io), to_dev(d, io)
    store = torch.empty(130 * far, dtype=t["q"].dtype, device="cuda")
    room = iter(range(0, 4096, 64))

    def spread(a=None):
        o = store.as_strided((1, 1, 130, 64), (130 * far, 130 * far, far, 1), next(room))
        return o if a is None else o.copy_(a)

    gates = (t["eta"], t["log_gamma"])
    out, w_out, ws = e2ttt.delta_forward(cfg, t["q"], t["k"], t["v"], *gates, t["w_in"], save_for_backward=True)
    g = e2ttt.delta_backward(cfg, t["q"], t["k"], t["v"], *gates, ws, td["d_out"], td["d_w_out"])
    q, k, v, do = [spread(a) for a in (t["q"], t["k"], t["v"], td["d_out"])]
    far_out, far_w, ws = e2ttt.delta_forward(cfg, q, k, v, *gates, t["w_in"], out=spread(), save_for_backward=True)
    grads = dict({n: torch.empty_like(a) for n, a in g.items()}, dq=spread(), dk=spread(), dv=spread())
    e2ttt.delta_backward(cfg, q, k, v, *gates, ws, do, td["d_w_out"], grads=grads)
    assert torch.equal(far_out, out) and torch.equal(far_w, w_out)
    for n in g:
        assert torch.equal(grads[n], g[n]), n
    with pytest.raises(e2ttt.E2TTTError):
        e2ttt.delta_forward(cfg, store.as_strided((1, 1, 130, 64), (0, 0, far + 8, 1)), k, v, *gates, t["w_in"])
