"""The query/key preparation element by element, against 64 bits (float32 tensors)."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def test_silu_of_values_of_any_size():
    """SiLU keeps its relative accuracy for large negative values.  In units of 2^-23: the
    exponential 1, its first-order correction 1/2 and, at -87, 3/4 that it leaves out, the
    sum 1/2, the reciprocal 1, the product 1/2, 4 1/4 together; in the derivative, (1 + x (1 - sigma)) sigma, the factor in brackets cancels
    around x = -1.28 and is off by a few 2^-23 of 1 + |x|."""
    g = torch.Generator().manual_seed(1)
    x = torch.cat([(torch.rand(40000, generator=g) - 0.5) * 172.0, torch.randn(24768, generator=g),
                   -torch.linspace(0, 87, 768)])
    cfg = e2ttt.QKConfig(1, 1, 0, x.numel() // 64, 64, 0, e2ttt.DT_F32, e2ttt.QK_SILU)
    q = x.view(1, 1, -1, 64).cuda()
    y, _ = e2ttt.qk_forward(cfg, q, None)
    z = x.double()
    ref = (z * torch.sigmoid(z)).view(1, 1, -1, 64)
    err = ((y.double().cpu() - ref).abs() / ref.abs().clamp(min=2.0 ** -120)).max().item()
    print("silu %.2e" % err, flush=True)
    assert err <= 4.25 * 2.0 ** -23
    dx, _ = e2ttt.qk_backward(cfg, torch.ones_like(q), None, q)
    s = torch.sigmoid(z)
    err = ((dx.double().cpu().flatten() - s * (1 + z * (1 - s))).abs() / (s * (1 + z.abs()))).max().item()
    print("dsilu %.2e" % err, flush=True)
    assert err <= 6 * 2.0 ** -23


def test_silu_of_special_values():
    """Infinities and NaN as x / (1 + exp(-x)) gives them; zero stays zero."""
    x = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 200.0, -200.0, 1e30])
    cfg = e2ttt.QKConfig(1, 1, 0, 1, 8, 0, e2ttt.DT_F32, e2ttt.QK_SILU)
    y, _ = e2ttt.qk_forward(cfg, x.view(1, 1, 1, 8).cuda(), None)
    want = x / (1.0 + torch.exp(-x))
    assert torch.equal(y.cpu().flatten().nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("interleaved", [False, True])
def test_sines_and_cosines(interleaved):
    """Pairs (1, 0) turn into the cosine and the sine.  Each is off by the rounding of the
    angle to its quarter turn (at most 2^-25 below pi / 4), of the last sum (2^-25) and of the
    square and the terms below it (2^-25 together): 2^-23 is asked for."""
    B, T, d = 4, 700, 128
    flags = e2ttt.QK_INTERLEAVED if interleaved else 0
    cfg = e2ttt.QKConfig(B, 1, 0, T, d, d, e2ttt.DT_F32, flags)
    f, _ = e2ttt.rotary_frequencies(d, device="cpu")
    pos = torch.randint(0, 200000, (B, T), generator=torch.Generator().manual_seed(2))
    x = torch.zeros(B, 1, T, d)
    first = slice(0, d, 2) if interleaved else slice(0, d // 2)
    second = slice(1, d, 2) if interleaved else slice(d // 2, d)
    x[..., first] = 1.0
    y, _ = e2ttt.qk_forward(cfg, x.cuda(), None, f.cuda(), pos.cuda())
    y = y.double().cpu()
    angle = pos.double()[:, None, :, None] * f.double()
    for name, got, ref in (("cos", y[..., first], torch.cos(angle)), ("sin", y[..., second], torch.sin(angle))):
        err = (got - ref).abs().max().item()
        print("%s %.2e" % (name, err), flush=True)
        assert err <= 2.0 ** -23, name


def test_rows_of_zeros_at_the_smallest_eps():
    cfg = e2ttt.QKConfig(1, 1, 0, 1, 8, 0, e2ttt.DT_F32, e2ttt.QK_SILU | e2ttt.QK_UNIT, eps=2.0 ** -126)
    q = torch.zeros(1, 1, 1, 8, device="cuda")
    assert (e2ttt.qk_forward(cfg, q, None)[0] == 0).all()
    dx, _ = e2ttt.qk_backward(cfg, torch.ones_like(q), None, q)
    # (half of 2^63: an ulp of the reciprocal root, of the reciprocal and two roundings)
    assert ((dx / 2.0 ** 62 - 1).abs() <= 4 * 2.0 ** -23).all()
