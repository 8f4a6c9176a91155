"""The delta rule with the gates that its interface allows but layers seldom make."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
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
