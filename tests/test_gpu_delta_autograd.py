"""The autograd wrappers of the delta rule and the query/key preparation with the
upstream gradients that a graph may hand them."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests.test_gpu_delta import make, to_dev

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "eta", "log_gamma", "w_in")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def shifted(t, n):
    """t as a contiguous tensor that starts n elements into its storage."""
    s = torch.empty(t.numel() + n, dtype=t.dtype, device=t.device)
    o = s[n:].view(t.shape)
    assert o.is_contiguous()
    return o.copy_(t)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_gradients_at_any_offset(io, layout):
    """Contiguous upstream gradients that do not start on 16 bytes, against aligned copies."""
    B, HK, H, T, d = 2, 1, 2, 70, 64
    x, up = make(B, HK, H, T, d, d, io, seed=91)
    code = e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32
    cfg = e2ttt.DeltaConfig(B, HK, H, T, d, d, code, 0.125)
    t = {n: a.requires_grad_(True) for n, a in to_dev(x, io, layout).items()}
    u = to_dev(up, io)
    out, w_out = e2ttt.DeltaFunction.apply(cfg, *[t[n] for n in NAMES])
    grads = lambda a, b: torch.autograd.grad([out, w_out], list(t.values()), [a, b], retain_graph=True)
    ref = grads(u["d_out"], u["d_w_out"])
    for n in (1, 3, 8):
        off = shifted(u["d_out"], n), shifted(u["d_w_out"], n)
        for got in (grads(*off), grads(off[0], u["d_w_out"]), grads(u["d_out"], off[1])):
            assert all(torch.equal(a, b) for a, b in zip(got, ref)), n
    qk = e2ttt.QKConfig(B, H, HK, T, d, d, code)
    f, _ = e2ttt.rotary_frequencies(d)
    q, k = [t[n].detach().requires_grad_(True) for n in ("v", "k")]
    qo, ko = e2ttt.QKFunction.apply(qk, q, k, f)
    grads = lambda a, b: torch.autograd.grad([qo, ko], [q, k], [a, b], retain_graph=True)
    d_k = u["d_out"][:, :1].contiguous()
    ref = grads(u["d_out"], d_k)
    for n in (1, 3, 8):
        for got in (grads(shifted(u["d_out"], n), shifted(d_k, n)), grads(u["d_out"], shifted(d_k, n))):
            assert all(torch.equal(a, b) for a, b in zip(got, ref)), n


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_gradients_through_a_concatenation(io):
    """A loss over one tensor of several parts hands back views at odd offsets."""
    c = (1, 1, 1, 70, 32, 32)
    x, _ = make(*c, io, seed=92)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 1.0)
    t = {n: a.requires_grad_(True) for n, a in to_dev(x, io).items()}
    aux = torch.ones(1, dtype=t["q"].dtype, device="cuda")
    out, w_out = e2ttt.DeltaFunction.apply(cfg, *[t[n] for n in NAMES])
    weight = torch.randn(1 + out.numel(), device="cuda").to(out.dtype)
    state = torch.randn(1 + w_out.numel(), device="cuda")
    loss = (torch.cat([aux, out.flatten()]) * weight).sum().float() + \
        (torch.cat([aux.float(), w_out.flatten()]) * state).sum()
    got = torch.autograd.grad(loss, list(t.values()), retain_graph=True)
    ref = torch.autograd.grad([out, w_out], list(t.values()),
                              [weight[1:].clone().view_as(out), state[1:].clone().view_as(w_out)])
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_nothing_saved_without_a_gradient():
    """Where no gradient can be asked for, the wrapper's call keeps nothing for one."""
    c = (1, 4, 4, 8192, 64, 64)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 0.125)
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    unit = lambda a: (a / a.norm(dim=-1, keepdim=True)).bfloat16()
    q, k, v = unit(rn(*c[:1], 4, 8192, 64)), unit(rn(*c[:1], 4, 8192, 64)), rn(1, 4, 8192, 64).bfloat16()
    rest = torch.sigmoid(rn(1, 4, 8192)), -0.1 * torch.rand(1, 4, 8192, device="cuda", generator=g), \
        rn(1, 4, 64, 64)

    def peak(v):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got = e2ttt.DeltaFunction.apply(cfg, q, k, v, *rest)
        return got, torch.cuda.max_memory_allocated() - before

    need = e2ttt.delta_workspace_bytes(cfg, True)
    leaf = v.clone().requires_grad_(True)
    ref, used = peak(leaf)
    assert used >= need and ref[0].requires_grad and ref[1].requires_grad
    plain, used = peak(v)
    assert used < need
    with torch.no_grad():
        quiet, also = peak(leaf)
    assert also < need
    for got in (plain, quiet):
        assert not got[0].requires_grad and not got[1].requires_grad
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    (dv,) = torch.autograd.grad(ref[0].float().sum(), leaf)
    assert torch.isfinite(dv).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_broadcast_inputs(io):
    """Inputs expanded over sequences, heads or tokens (strides of 0) give what their copies
    give, gradients of the leaves among them."""
    B, HK, H, T, d = 2, 1, 2, 90, 32
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    cfg = e2ttt.DeltaConfig(B, HK, H, T, d, d, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32, 1.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    leaves = [a.requires_grad_(True) for a in (
        unit(rn(1, 1, T, d)).to(dt), unit(rn(B, 1, 1, d)).to(dt), rn(B, 1, T, d).to(dt),
        torch.sigmoid(rn(1, H, 1)), -torch.sigmoid(rn(B, 1, T)))]
    shapes = [(B, HK, T, d)] * 2 + [(B, H, T, d)] + [(B, H, T)] * 2

    def step(copy):
        a = [t.expand(s) for t, s in zip(leaves, shapes)]
        assert not any(t.is_contiguous() for t in a)
        out, w = e2ttt.DeltaFunction.apply(cfg, *[t.contiguous() if copy else t for t in a])
        return [out, w, *torch.autograd.grad((out.float() ** 2).sum() + w.sum(), leaves)]

    assert all(torch.equal(a, b) for a, b in zip(step(False), step(True)))
