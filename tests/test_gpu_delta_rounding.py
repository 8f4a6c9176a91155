"""The delta rule's bf16 outputs and gradients are fp32 results rounded once.

They are compared with the 64-bit recurrence rounded to bf16.  An fp32 value
that is off by e_i falls on the other side of a rounding border with
probability |e_i| / u_i, where u_i <= 2^-7 |x_i| is the distance of neighbouring
bf16 numbers, and is then u_i off.  The expected square of the difference is
sum |e_i| u_i <= |e| |u| <= 2^-7 |e| |x|, which with the |e| <= 2^-18 |x| that is
asked of fp32 results (test_gpu_delta.py) is (2^-12.5 |x|)^2; 2^-12 |x| is asked
for, over tensors of 10^4 elements and more.  (Products of operands of two bf16
parts, off by 2^-15, give 2^-11.)"""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import deltaref
from tests.test_gpu_delta import make, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def rounded_once(name, got, ref):
    want = ref.bfloat16().double()
    assert want.numel() >= 10000
    err = ((got.double().cpu() - want).norm() / want.norm()).item()
    print("%-4s %.2e" % (name, err), flush=True)
    assert err <= 2.0 ** -12, (name, err)


@pytest.mark.parametrize("c", [(2, 1, 2, 200, 64, 64),       # chunks in turn
                               (1, 2, 2, 801, 32, 40),       # segments
                               (1, 1, 2, 600, 128, 72),
                               (4, 24, 24, 2049, 64, 8)])    # parts
def test_rounded_once(c):
    B, HK, H, T, dk, dv = c
    x, d = make(*c, "bf16", seed=83)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 0.125)
    t, td = to_dev(x, "bf16"), to_dev(d, "bf16")
    names = ("q", "k", "v", "eta", "log_gamma")
    print("delta", c, flush=True)
    out, _, ws = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"], save_for_backward=True)
    plain, _, _ = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"])
    g = e2ttt.delta_backward(cfg, *[t[n] for n in names], ws, td["d_out"], td["d_w_out"])
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
    one = lambda a: a[:1]          # (the sequences do not meet)
    ref, _, rg = deltaref.delta_grads({n: one(a) for n, a in x.items()}, 0.125, one(d["d_out"]),
                                      one(d["d_w_out"]))
    for name, got, want in (("out", out, ref), ("dq", g["dq"], rg["q"]), ("dk", g["dk"], rg["k"]),
                            ("dv", g["dv"], rg["v"])):
        rounded_once(name, one(got), want)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_f32_states_stay_f32_between_segments(io):
    """The state goes from segment to segment in float32.  With eta = 0 it decays by 1 - 2^-20
    once in each of 16 segments; states just below 2 and that factor have mantissas of ones,
    of which a product of cut off bf16 terms leaves out 2^-23 every time (2^-19 in all).  Asked for: the exponential an ulp (2^-24) off, 16 times, and the products'
    independent roundings, sqrt(16) 2^-24."""
    B, H, T, d = 1, 1, 4096, 64
    g = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=g).cuda()
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    cfg = e2ttt.DeltaConfig(B, H, H, T, d, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 1.0)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    q, k, v = unit(rn(B, H, T, d)).to(dt), unit(rn(B, H, T, d)).to(dt), rn(B, H, T, d).to(dt)
    eta, lg = torch.zeros(B, H, T, device="cuda"), torch.zeros(B, H, T, device="cuda")
    lg[:, :, 100::256] = -2.0 ** -20
    ones = 2.0 - 2.0 ** -23 * torch.randint(1, 256, (B, H, d, d), generator=g).float().cuda()
    _, w_out, ws = e2ttt.delta_forward(cfg, q, k, v, eta, lg, ones, save_for_backward=True)
    grads = e2ttt.delta_backward(cfg, q, k, v, eta, lg, ws, torch.zeros_like(v), ones)
    ref = ones.double() * torch.exp(lg.double().sum())
    for name, got in (("w_out", w_out), ("d_w_in", grads["d_w_in"])):
        err = ((got.double() - ref).norm() / ref.norm()).item()
        print("%-6s %.2e" % (name, err), flush=True)
        assert err <= 2.0 ** -20 + 2.0 ** -22, (name, err)
