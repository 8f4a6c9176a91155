"""The delta rule with the gates that its interface allows but layers seldom make."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import deltaref
from tests.test_gpu_delta import close, make, to_dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_decays_to_nothing_and_back(io):
    """A decay below what fp32 holds and growth after it in the same chunk: a state that takes
    no updates comes back as e^-120 e^40 e^40 of itself, and after a decay of -inf it does
    not come back."""
    c = (1, 1, 2, 100, 32, 32)
    x, d = make(*c, io, seed=95)
    x["eta"][:] = 0.0
    x["log_gamma"][:] = 0.0
    x["log_gamma"][:, 0, 20] = -120.0
    x["log_gamma"][:, 1, 20] = -float("inf")
    x["log_gamma"][:, :, 22] = 40.0
    x["log_gamma"][:, :, 30] = 40.0
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 0.25)
    t, td = to_dev(x, io), to_dev(d, io)
    names = ("q", "k", "v", "eta", "log_gamma")
    out, w_out, ws = e2ttt.delta_forward(cfg, *[t[n] for n in names], t["w_in"], save_for_backward=True)
    g = e2ttt.delta_backward(cfg, *[t[n] for n in names], ws, torch.zeros_like(td["d_out"]), td["d_w_out"])
    big = 2.0 ** 57                # (2^57 e^-40: of the size that close() looks at)
    left = torch.exp(torch.tensor(-40.0, dtype=torch.float64)) * big
    read = lambda w, s: (0.25 * w @ x["q"][:, 0, s].transpose(-1, -2)).transpose(-1, -2)
    close("before", out[:, 0, :20], read(x["w_in"][:, 0], slice(0, 20)), io)
    close("after", out[:, 0, 30:] * big, left * read(x["w_in"][:, 0], slice(30, 100)), io)
    close("w_out", w_out[:, 0] * big, left * x["w_in"][:, 0], "f32")
    close("d_w_in", g["d_w_in"][:, 0] * big, left * d["d_w_out"][:, 0], "f32")
    dot = (x["w_in"][:, 0] * d["d_w_out"][:, 0]).sum()
    close("d_log_gamma", g["d_log_gamma"][:, 0] * big, (left * dot).expand(1, 100), "f32")
    for a in (out[:, 1, 20:], w_out[:, 1], g["d_w_in"][:, 1], g["d_log_gamma"][:, 1]):
        assert (a == 0).all()


def test_gates_of_the_framework():
    """The gate parameterisation's eta and gamma drive the rule through log(gamma)."""
    c = (2, 1, 2, 100, 32, 32)
    x, d = make(*c, "f32", seed=97)
    gen = torch.Generator().manual_seed(5)
    logits = [torch.randn(2, 2, 100, generator=gen) for _ in range(3)]
    params = dict(eta_base=0.9, alpha_base=0.5, tau=32.0)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_F32, 0.25)
    t, td = to_dev(x, "f32"), to_dev(d, "f32")
    leaves = [a.cuda().requires_grad_(True) for a in (logits[0], logits[2])]
    eta, _, gamma = e2ttt.GatesFunction.apply(e2ttt.GateParams(**params), leaves[0], logits[1].cuda(), leaves[1])
    out, w_out = e2ttt.DeltaFunction.apply(cfg, t["q"], t["k"], t["v"], eta, gamma.log(), t["w_in"])
    got = torch.autograd.grad([out, w_out], leaves, [td["d_out"], td["d_w_out"]])
    ref = [logits[0].double().requires_grad_(True), logits[2].double().requires_grad_(True)]
    r_eta = 0.9 * torch.sigmoid(ref[0])
    r_gamma = 1 - r_eta * 0.5 * torch.sigmoid(ref[1])
    ro, rw = deltaref.delta(x["q"], x["k"], x["v"], r_eta, r_gamma.log(), x["w_in"], 0.25)
    want = torch.autograd.grad([ro, rw], ref, [d["d_out"], d["d_w_out"]])
    # (gates to 2e-6 of their values and gradients to 1e-5, as their own tests ask)
    for n, a, b, tol in (("out", out, ro, 1e-5), ("w_out", w_out, rw, 1e-5), ("d_l_eta", got[0], want[0], 4e-5),
                         ("d_l_alpha", got[1], want[1], 4e-5)):
        err = ((a.detach().double().cpu() - b.detach()).norm() / b.detach().norm()).item()
        print("%-10s rel %.2e" % (n, err), flush=True)
        assert err <= tol, (n, err)
