"""Attention and the delta rule side by side on the same prepared queries, keys and
values, as a token-mixing block runs them: a training step, and serving (a prompt,
its cache, then token by token in a window).

Tolerances in the 2-norm.  Training: between a leaf's gradient and 64 bits lie at
most eight roundings to the io type (prepared row, probabilities, dS, out, the two
branches' gradients, their sum, the leaf's own), each of at most half a step: 8 x
2^-8, and with float32 8 x 2^-18 for what the sums of each add.  Serving compares
each branch on the rows that the card itself prepared."""
import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import attnref, cacheref, deltaref
from tests.test_gpu_attention import rounded
from tests.test_gpu_delta import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def near(name, got, ref, tol):
    err = ((got.detach().double().cpu() - ref).norm() / ref.norm()).item()
    print("%-8s rel %.2e" % (name, err), flush=True)
    assert err <= tol, (name, err)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_training_step(io):
    B, HK, H, T, d, W = 2, 2, 4, 150, 64, 48
    g = torch.Generator().manual_seed(6)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    lengths = torch.tensor([T, 90])
    x = dict(q=rounded(rn(B, H, T, d), io), k=rounded(rn(B, HK, T, d), io), v=rounded(rn(B, H, T, d), io),
             va=rounded(rn(B, HK, T, d), io), eta=torch.sigmoid(rn(B, H, T)).float().double(),
             g=(-0.1 * torch.rand(B, H, T, generator=g, dtype=torch.float64)).float().double())
    d_out = rounded(rn(B, H, T, d), io)
    fr, m = e2ttt.rotary_frequencies(d, device="cpu")
    pos = torch.arange(T).expand(B, T)

    # 64 bits.  (the rule's queries: one a key head, the first of its group)
    r = {n: t.clone().requires_grad_(True) for n, t in x.items()}
    prep = lambda t: deltaref.qk_row(t, fr, pos, d, True, True, False, 1e-6, m)
    q, k = prep(r["q"]), prep(r["k"])
    a, _, _ = attnref.attention(dict(q=q, k=k, v=r["va"]), 4.0, W - 1, 0, lengths)
    o, _ = deltaref.delta(q[:, ::H // HK], k, r["v"], r["eta"], r["g"],
                          torch.zeros(B, H, d, d, dtype=torch.float64), d ** -0.5, lengths)
    ref = dict(zip(r, torch.autograd.grad(((a + o) * d_out).sum(), list(r.values()))))

    E = e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32
    t = {n: dev(y, io if n in ("q", "k", "v", "va") else "f32").requires_grad_(True) for n, y in x.items()}
    tl = lengths.to(torch.int32).cuda()
    qc = e2ttt.QKConfig(B, H, HK, T, d, d, E, rot_scale=m)
    ac = e2ttt.AttentionConfig(B, HK, H, T, d, E, scale=4.0, left=W - 1)
    dc = e2ttt.DeltaConfig(B, HK, H, T, d, d, E, scale=d ** -0.5)
    q, k = e2ttt.QKFunction.apply(qc, t["q"], t["k"], fr.cuda())
    a1, _ = e2ttt.AttentionFunction.apply(ac, q, k, t["va"], tl)
    o1, _ = e2ttt.DeltaFunction.apply(dc, q[:, ::H // HK], k, t["v"], t["eta"], t["g"], None, tl)
    got = torch.autograd.grad(((a1 + o1) * dev(d_out, io)).sum(), list(t.values()))
    tol = 8 * 2.0 ** (-8 if io == "bf16" else -18)
    near("out", a1 + o1, (a + o).detach(), tol)
    for n, y in zip(t, got):
        near("d_" + n, y, ref[n], tol)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_prompt_then_tokens(io):
    """A prompt through attention and the rule, its last window into a ring of pages,
    then tokens one and three at a time from the cache and the state."""
    B, HK, H, d, W, T0 = 2, 2, 4, 64, 100, 170
    steps = [1, 1, 3, 1, 2, 1, 1]
    n = T0 + sum(steps)
    g = torch.Generator().manual_seed(8)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    E = e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32
    fr, m = e2ttt.rotary_frequencies(d, device="cpu")
    x = {a: dev(rounded(rn(B, h, n, d), io), io) for a, h in (("q", H), ("k", HK), ("v", HK))}
    q, k = e2ttt.qk_forward(e2ttt.QKConfig(B, H, HK, n, d, d, E, rot_scale=m), x["q"], x["k"], fr.cuda())
    v = x["v"]
    host = {a: y.double().cpu() for a, y in (("q", q), ("k", k), ("v", v))}

    # the prompt: exact keys; what it leaves: the cache's
    cut = lambda y, a, b: y[:, :, a:b]
    cfg = e2ttt.AttentionConfig(B, HK, H, T0, d, E, scale=4.0, left=W - 1)
    o, _ = e2ttt.attention_forward(cfg, *(cut(y, 0, T0) for y in (q, k, v)))
    ref, _, _ = attnref.attention({a: cut(y, 0, T0) for a, y in host.items()}, 4.0, W - 1, 0, None)
    tol = 2.0 ** (-8 if io == "bf16" else -18)
    near("prompt", o, ref, tol)
    P, pages = 3, 2 * 3 + 2          # (a ring of 192 tokens for a window of 100)
    table = torch.randperm(pages, generator=g)[:2 * P].view(2, P).to(torch.int32).cuda()
    cc = lambda T: e2ttt.CacheConfig(B, HK, H, T, d, P, E, scale=4.0, left=W - 1)
    cache = e2ttt.alloc_cache(cc(1), pages)
    e2ttt.cache_write(cc(T0), cut(k, 0, T0), cut(v, 0, T0), cache, table)
    kv = list(zip(*(cacheref.values(*cacheref.quantise(host[a])) for a in ("k", "v"))))
    state = torch.zeros(B, HK, d, d, device="cuda")
    eta = torch.sigmoid(rn(B, HK, n)).float().cuda()
    w = torch.zeros(B, HK, d, d, dtype=torch.float64)
    rule = lambda T: e2ttt.DeltaConfig(B, HK, HK, T, d, d, E, scale=d ** -0.5)
    qr = q[:, ::H // HK]
    _, state, _ = e2ttt.delta_forward(rule(T0), cut(qr, 0, T0), cut(k, 0, T0), cut(v, 0, T0),
                                      eta[:, :, :T0])
    t = T0
    for s in steps:
        at = torch.full((B,), t, dtype=torch.int32, device="cuda")
        e2ttt.cache_write(cc(s), cut(k, t, t + s), cut(v, t, t + s), cache, table, at)
        a, _ = e2ttt.cache_attention(cc(s), cut(q, t, t + s), cache, table, at)
        r = e2ttt.delta_step(rule(s), cut(qr, t, t + s), cut(k, t, t + s), cut(v, t, t + s),
                             eta[:, :, t:t + s].contiguous(), None, state)
        ref, _, _ = cacheref.attend(cut(host["q"], t, t + s), kv, [t] * B, [s] * B, P, W - 1, 4.0)
        near("tokens", a, ref, tol)
        t += s
        assert torch.isfinite(r).all()
    ref, w = deltaref.delta(host["q"][:, ::H // HK], host["k"], host["v"], eta.double().cpu(), None, w,
                            d ** -0.5)
    near("rule", r, cut(ref, t - steps[-1], t), tol)
    near("state", state, w, 2.0 ** -18)
    # the window read back is what the next segment's attention would stand on
    back, _ = e2ttt.cache_read(cc(W), cache, table, torch.full((B,), n - W, dtype=torch.int32, device="cuda"))
    assert torch.equal(back.double().cpu(), torch.stack([a[:, n - W:] for a, _ in kv]))
