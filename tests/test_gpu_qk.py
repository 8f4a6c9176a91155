"""GPU parity of the query/key preparation with its formulas in 64 bits
(tests/deltaref.py).  An element passes a handful of fp32 roundings (2^-24
each; the row sum of up to 256 squares another 16) and, with bf16, one of at
most 2^-8 of its value: 2^-8 + 2^-16 and 2^-18 in the 2-norm of a tensor."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import deltaref
from tests.test_gpu_delta import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def close(name, got, ref, io):
    got = got.double().cpu()
    err, n = (got - ref).norm().item(), ref.norm().item()
    print("%-4s rel %.2e" % (name, err / max(n, 1e-30)), flush=True)
    assert err <= (2.0 ** -8 + 2.0 ** -16 if io == "bf16" else 2.0 ** -18) * n, (name, err / n)


def inputs(B, H, HK, T, d, io, seed):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    rn = lambda h: torch.randn(B, h, T, d, generator=g, dtype=torch.float64).to(dt).double()
    return rn(H), rn(HK), rn(H), rn(HK)


CASES = [  # B, H, HK, T, d, rot
    (1, 1, 1, 1, 8, 8), (2, 3, 1, 5, 16, 0), (2, 4, 2, 33, 64, 64), (1, 2, 2, 7, 64, 34),
    (3, 2, 1, 9, 128, 48), (1, 5, 5, 17, 256, 254), (2, 1, 1, 3, 256, 6), (1, 2, 1, 40, 72, 36),
    (1, 2, 1, 6, 96, 2), (1, 1, 1, 11, 200, 100)]


@pytest.mark.parametrize("c", CASES)
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("flags", range(8))
def test_forward_backward(c, io, flags):
    B, H, HK, T, d, rot = c
    q, k, gq, gk = inputs(B, H, HK, T, d, io, 7 * flags + d)
    if T > 2:
        q[0, 0, 2] = 0.0           # a row of zeros stays one
    layout = "bthd" if flags & 1 else "bhtd"
    pos = torch.randint(0, 100000, (B, T), generator=torch.Generator().manual_seed(d))
    fr, m = e2ttt.rotary_frequencies(rot, device="cpu")
    m = 1.25 if flags & 2 else m
    cfg = e2ttt.QKConfig(B, H, HK, T, d, rot, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, flags,
                         rot_scale=m)
    print("qk", c, io, flags, flush=True)
    tq, tk = dev(q, io, layout), dev(k, io, layout)
    tg, th = dev(gq, io, layout), dev(gk, io, layout)
    inv = fr.cuda() if rot else None
    qo, ko = e2ttt.qk_forward(cfg, tq, tk, inv, pos.cuda())
    need = flags & 3
    dq, dk = e2ttt.qk_backward(cfg, tg, th, tq if need else None, tk if need else None, inv, pos.cuda())
    args = (fr, pos, rot, bool(flags & 1), bool(flags & 2), bool(flags & 4), 1e-6, m)
    for name, x, g, y, dx in (("q", q, gq, qo, dq), ("k", k, gk, ko, dk)):
        x = x.clone().requires_grad_(True)
        ref = deltaref.qk_row(x, *args)
        (rd,) = torch.autograd.grad(ref, x, g)
        close(name, y, ref.detach(), io)
        close("d" + name, dx, rd, io)
        # and the gradient against a central difference of the 64-bit formula
        u = torch.randn(x.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        h = 1e-6
        with torch.no_grad():
            num = (((deltaref.qk_row(x + h * u, *args) - deltaref.qk_row(x - h * u, *args)) * g).sum() / (2 * h)).item()
        tol = 2.0 ** -8 if io == "bf16" else 2.0 ** -18
        # (rows of zeros under the unit length curve at the scale of sqrt(eps) = 1e-3: h^2 / eps)
        assert abs((dx.double().cpu() * u).sum().item() - num) <= \
            2 * tol * rd.norm().item() * u.norm().item() + 1e-5 * abs(num)
    # in place, the keys left out, and positions 0 .. T - 1 by default
    buf = (tq.clone(memory_format=torch.preserve_format), tk.clone(memory_format=torch.preserve_format))
    e2ttt.qk_forward(cfg, *buf, inv, pos.cuda(), out=buf)
    assert torch.equal(buf[0], qo) and torch.equal(buf[1], ko)
    alone = e2ttt.QKConfig(B, H, 0, T, d, rot, cfg.io, flags, rot_scale=m)
    assert torch.equal(e2ttt.qk_forward(alone, tq, None, inv, pos.cuda())[0], qo)
    first = torch.arange(T).repeat(B, 1).cuda()
    a, b = e2ttt.qk_forward(cfg, tq, tk, inv), e2ttt.qk_forward(cfg, tq, tk, inv, first)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_far_positions():
    """Angles at positions where 32 bits hold no fraction of a turn."""
    cfg = e2ttt.QKConfig(1, 1, 1, 4, 64, 64, e2ttt.DT_F32, 0)
    q, k, _, _ = inputs(1, 1, 1, 4, 64, "f32", 1)
    pos = torch.tensor([[2 ** 24 + 1, 2 ** 31 + 12345, 2 ** 40 + 7, -5]])
    fr, _ = e2ttt.rotary_frequencies(64, device="cpu")
    qo, ko = e2ttt.qk_forward(cfg, dev(q, "f32"), dev(k, "f32"), fr.cuda(), pos.cuda())
    # the 64-bit angle itself is off by 2^-53 of 2^40: 2^-13 of a radian at the last but one
    for i, tol in enumerate((2.0 ** -18, 2.0 ** -18, 2.0 ** -11, 2.0 ** -18)):
        for x, y in ((q, qo), (k, ko)):
            ref = deltaref.qk_row(x, fr, pos, 64, False, False, False, 1e-6, 1.0)[:, :, i]
            assert (y[:, :, i].double().cpu() - ref).norm() <= tol * ref.norm(), i


def test_heads_of_a_group_share_angles():
    """Many tokens (several heads to a group of lanes), an odd number of heads."""
    B, H, HK, T, d = 2, 7, 4, 4100, 64
    cfg = e2ttt.QKConfig(B, H, HK, T, d, 64, e2ttt.DT_BF16, e2ttt.QK_SILU | e2ttt.QK_UNIT)
    q, k, _, _ = inputs(B, H, HK, T, d, "bf16", 5)
    fr, _ = e2ttt.rotary_frequencies(64, device="cpu")
    pos = torch.arange(T).repeat(B, 1)
    for layout in ("bhtd", "bthd"):
        qo, ko = e2ttt.qk_forward(cfg, dev(q, "bf16", layout), dev(k, "bf16", layout), fr.cuda())
        close("q", qo, deltaref.qk_row(q, fr, pos, 64, True, True, False, 1e-6, 1.0), "bf16")
        close("k", ko, deltaref.qk_row(k, fr, pos, 64, True, True, False, 1e-6, 1.0), "bf16")


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_layer(io):
    """As they are used together: preparation, the delta rule, and their backward; and the
    same preparation ahead of the framework's chunk update."""
    B, H, T, d = 2, 2, 100, 64
    g = torch.Generator().manual_seed(9)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x = dict(q=rn(B, H, T, d), k=rn(B, H, T, d), v=rn(B, H, T, d))
    x = {n: a.to(dt).double() for n, a in x.items()}
    x["eta"], x["log_gamma"] = torch.sigmoid(rn(B, H, T)).float().double(), -0.1 * torch.rand(B, H, T, generator=g).double()
    d_out = rn(B, H, T, d).to(dt).double()
    t = {n: dev(a, io if n in "qkv" else "f32").requires_grad_(True) for n, a in x.items()}
    code = e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32
    qcfg = e2ttt.QKConfig(B, H, H, T, d, d, code)
    dcfg = e2ttt.DeltaConfig(B, H, H, T, d, d, code, d ** -0.5)
    fr, _ = e2ttt.rotary_frequencies(d)
    qp, kp = e2ttt.QKFunction.apply(qcfg, t["q"], t["k"], fr)
    out, _ = e2ttt.DeltaFunction.apply(dcfg, qp, kp, t["v"], t["eta"], t["log_gamma"])
    grads = torch.autograd.grad(out, list(t.values()), dev(d_out, io))
    y = {n: a.clone().requires_grad_(True) for n, a in x.items()}
    y["log_gamma"] = t["log_gamma"].detach().double().cpu().requires_grad_(True)
    pos = torch.arange(T).repeat(B, 1)
    prep = lambda a: deltaref.qk_row(a, fr.cpu(), pos, d, True, True, False, 1e-6, 1.0)
    ro, _ = deltaref.delta(prep(y["q"]), prep(y["k"]), y["v"], y["eta"], y["log_gamma"],
                           torch.zeros(B, H, d, d, dtype=torch.float64), d ** -0.5)
    rg = torch.autograd.grad(ro, list(y.values()), d_out)
    # bf16: q', k' and their gradients are rounded between the two operators, 2^-8 each, and
    # what a changed key changes passes the rule's solve (a few times the relative change)
    tol = 16 * 2.0 ** -8 if io == "bf16" else 2.0 ** -16
    for n, a, r in [("out", out.detach(), ro.detach())] + list(zip(y, grads, rg)):
        err = ((a.double().cpu() - r).norm() / r.norm()).item()
        print("layer", io, n, "%.2e" % err, flush=True)
        assert err <= tol, (n, err)
    if io == "bf16":
        cfg = e2ttt.Config(B, H, T, d, 64, 64)
        w = 0.02 * torch.randn(B, H, cfg.P, device="cuda")
        beta = torch.full_like(t["eta"], 0.9).detach()
        a = e2ttt.forward(cfg, qp.detach(), kp.detach(), t["v"].detach(), 0.01 * t["eta"].detach(),
                          beta, None, w)[0]
        assert torch.isfinite(a).all()
