"""The delta rule's and the query/key preparation's ways of filling the card that
small calls do not take: eight waves a workgroup, segments and parts captured and
on other streams, parts within stretches, several heads to a group of lanes."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import deltaref
from tests.test_gpu_delta import close, make, to_dev
from tests.test_gpu_qk import close as close_qk

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "eta", "log_gamma")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def random_call(c, seed, rate=0.1):
    """Inputs of a call of c on the GPU, of bf16 tensors."""
    B, HK, H, T, dk, dv = c
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)
    unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).bfloat16()
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, dk ** -0.5)
    x = dict(q=unit(rn(B, HK, T, dk)), k=unit(rn(B, HK, T, dk)), v=rn(B, H, T, dv).bfloat16(),
             eta=torch.sigmoid(rn(B, H, T)), log_gamma=-rate * torch.rand(B, H, T, device="cuda", generator=g),
             w_in=0.3 * rn(B, H, dv, dk))
    return cfg, x, dict(d_out=rn(B, H, T, dv).bfloat16(), d_w_out=0.3 * rn(B, H, dv, dk))


# 32 units of 128 x 128 in segments (more than 128 workgroups of eight waves; the state passes
# too), and 136 units whose chunks run in turn.
@pytest.mark.parametrize("c,lengths", [((2, 16, 16, 1088, 128, 128), (1088, 900)),
                                       ((17, 8, 8, 130, 128, 128), None),
                                       ((17, 4, 8, 70, 72, 128), None)])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_eight_waves(c, lengths, layout):
    B, HK, H, T, dk, dv = c
    x, d = make(*c, "bf16", seed=101, rate=0.02)
    cfg = e2ttt.DeltaConfig(*c, e2ttt.DT_BF16, 0.125)
    t, td = to_dev(x, "bf16", layout), to_dev(d, "bf16", layout)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    lg = None if ln is None else ln.cuda()
    print("delta", c, layout, flush=True)
    out, w_out, ws = e2ttt.delta_forward(cfg, *[t[n] for n in NAMES], t["w_in"], lengths=lg,
                                         save_for_backward=True)
    g = e2ttt.delta_backward(cfg, *[t[n] for n in NAMES], ws, td["d_out"], td["d_w_out"], lengths=lg)
    w = t["w_in"].clone()
    out2, _, _ = e2ttt.delta_forward(cfg, *[t[n] for n in NAMES], w, lengths=lg, w_out=w)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(w_out, w)
    rep = H // HK
    for b, hk in ((0, 0), (B - 1, HK - 1)):     # (key heads with their value heads do not meet)
        def one(a, n):
            h = slice(hk, hk + 1) if n in ("q", "k", "dq", "dk") else slice(rep * hk, rep * (hk + 1))
            return a[b:b + 1, h]
        ro, rw, rg = deltaref.delta_grads({n: one(a, n) for n, a in x.items()}, 0.125,
                                          one(d["d_out"], "v"), one(d["d_w_out"], "v"),
                                          None if ln is None else ln[b:b + 1])
        close("out", one(out, "v"), ro, "bf16")
        close("w_out", one(w_out, "v"), rw, "f32")
        for n, m, ty in (("q", "dq", "bf16"), ("k", "dk", "bf16"), ("v", "dv", "bf16"),
                         ("eta", "d_eta", "f32"), ("log_gamma", "d_log_gamma", "f32"),
                         ("w_in", "d_w_in", "f32")):
            close(m, one(g[m], m), rg[n], ty)


def test_parts_within_stretches():
    """Without saving, 128 units take long sequences in several stretches, each in parts, and
    carry their state from launch to launch: bit for bit the saving call (one stretch) and the
    calls of the sequence's halves; and the recurrence, for one unit."""
    c = (8, 16, 16, 12800, 64, 64)
    cfg, x, _ = random_call(c, 7, rate=0.003)
    each = e2ttt.delta_workspace_bytes(e2ttt.DeltaConfig(8, 16, 16, 64, 64, 64), False)
    assert e2ttt.delta_workspace_bytes(cfg, False) < 150 * each       # (200 chunks)
    a = [x[n] for n in NAMES]
    out, w_out, _ = e2ttt.delta_forward(cfg, *a, x["w_in"])
    saved, w_saved, ws = e2ttt.delta_forward(cfg, *a, x["w_in"], save_for_backward=True)
    assert torch.equal(saved, out) and torch.equal(w_saved, w_out)
    del ws, saved
    half = e2ttt.DeltaConfig(8, 16, 16, 6400, 64, 64, e2ttt.DT_BF16, cfg.scale)
    o1, w, _ = e2ttt.delta_forward(half, *[t[:, :, :6400] for t in a], x["w_in"])
    o2, _, _ = e2ttt.delta_forward(half, *[t[:, :, 6400:] for t in a], w, w_out=w)
    assert torch.equal(torch.cat([o1, o2], 2), out) and torch.equal(w, w_out)
    one = {n: t[7:8, 15:16].double().cpu() for n, t in x.items()}
    ro, rw = deltaref.delta(*[one[n] for n in NAMES], one["w_in"], cfg.scale)
    close("out", out[7:8, 15:16], ro, "bf16")
    close("w_out", w_out[7:8, 15:16], rw, "f32")


def test_few_units_against_many():
    """A sequence among many (its chunks in turn, in stretches) and alone (in segments)."""
    c = (64, 8, 32, 64 * 12, 16, 16)
    cfg, x, d = random_call(c, 11)
    few = e2ttt.DeltaConfig(1, *c[1:], e2ttt.DT_BF16, cfg.scale)
    a, one = [x[n] for n in NAMES], [x[n][:1].contiguous() for n in NAMES]
    out, w, ws = e2ttt.delta_forward(cfg, *a, x["w_in"], save_for_backward=True)
    g = e2ttt.delta_backward(cfg, *a, ws, d["d_out"], d["d_w_out"])
    o1, w1, ws = e2ttt.delta_forward(few, *one, x["w_in"][:1].contiguous(), save_for_backward=True)
    g1 = e2ttt.delta_backward(few, *one, ws, d["d_out"][:1].contiguous(), d["d_w_out"][:1].contiguous())
    close("out", out[:1], o1.double().cpu(), "bf16")
    close("w_out", w[:1], w1.double().cpu(), "f32")
    for n in g:
        close(n, g[n][:1], g1[n].double().cpu(), "bf16" if n in ("dq", "dk", "dv") else "f32")


# in segments (64: chunks of 64 x 64; 128: eight waves), and in parts
@pytest.mark.parametrize("c", [(1, 1, 2, 1500, 64, 64), (2, 8, 16, 1088, 128, 128),
                               (8, 8, 16, 2100, 64, 64)])
def test_captured_and_on_other_streams(c):
    """A training step on another stream, on two streams at once and as a graph, replayed with
    eager work between the replays, equals the eager step on the default stream."""
    cfg, x, d = random_call(c, 13)

    class Step:
        def __init__(self):
            self.ws = e2ttt.alloc_delta_workspace(cfg, True)
            self.sc = torch.empty(e2ttt.delta_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
            self.out, self.w = torch.empty_like(x["v"]), torch.empty_like(x["w_in"])
            self.g = dict(dq=torch.empty_like(x["q"]), dk=torch.empty_like(x["k"]),
                          dv=torch.empty_like(x["v"]), d_eta=torch.empty_like(x["eta"]),
                          d_log_gamma=torch.empty_like(x["eta"]), d_w_in=torch.empty_like(x["w_in"]))

        def run(self):
            a = [x[n] for n in NAMES]
            e2ttt.delta_forward(cfg, *a, x["w_in"], out=self.out, w_out=self.w, workspace=self.ws,
                                save_for_backward=True)
            e2ttt.delta_backward(cfg, *a, self.ws, d["d_out"], d["d_w_out"], grads=self.g,
                                 scratch=self.sc)

        def results(self):
            return [self.out, self.w, *self.g.values()]

    one, two = Step(), Step()
    one.run()
    torch.cuda.synchronize()
    ref = [t.clone() for t in one.results()]
    same = lambda s: all(torch.equal(t, r) for t, r in zip(s.results(), ref))

    def clear(*steps):
        for s in steps:
            for t in s.results():
                t.fill_(float("nan"))

    streams = torch.cuda.Stream(), torch.cuda.Stream()
    clear(one, two)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, step in zip(streams, (one, two)):
            with torch.cuda.stream(s):
                step.run()
    torch.cuda.synchronize()
    assert same(one) and same(two)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.run()
    for i in range(4):
        clear(one, two)
        graph.replay()
        two.run()
        torch.cuda.synchronize()
        assert same(one) and same(two), i
        one.run()
        torch.cuda.synchronize()
        assert same(one), i


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_heads_share_a_group_of_lanes(io, layout):
    """48,000 tokens of 7 + 4 heads: four (bf16) and eight (f32) heads to a group of lanes, a
    group with query and key heads, and a last one that is not full; forward and backward."""
    B, H, HK, T, d, rot = 2, 7, 4, 24000, 64, 64
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    cfg = e2ttt.QKConfig(B, H, HK, T, d, rot, e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32)
    g = torch.Generator(device="cuda").manual_seed(17)

    def rn(h):
        t = torch.randn(B, h, T, d, device="cuda", generator=g).to(dt)
        return t.transpose(1, 2).contiguous().transpose(1, 2) if layout == "bthd" else t

    q, k, dq, dk = rn(H), rn(HK), rn(H), rn(HK)
    f, _ = e2ttt.rotary_frequencies(rot)
    pos = torch.randint(0, 100000, (B, T), device="cuda", generator=g)
    qo, ko = e2ttt.qk_forward(cfg, q, k, f, pos)
    gq, gk = e2ttt.qk_backward(cfg, dq, dk, q, k, f, pos)
    for name, x, up, y, gx in (("q", q, dq, qo, gq), ("k", k, dk, ko, gk)):
        x = x.double().requires_grad_(True)
        ref = deltaref.qk_row(x, f, pos, rot, True, True, False, 1e-6, 1.0)
        (rg,) = torch.autograd.grad(ref, x, up.double())
        for h in range(x.shape[1]):              # (each head: none may be another's)
            close_qk(name + str(h), y[:, h], ref[:, h].detach().cpu(), io)
            close_qk("d" + name + str(h), gx[:, h], rg[:, h].cpu(), io)
