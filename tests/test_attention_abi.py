"""Refusals and sizes of the attention entry points, and the reference that the GPU
tests compare with; no call here reaches a kernel."""
import ctypes
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import attnref


@pytest.fixture(scope="module")
def lib():
    return e2ttt.load()


FAKE = ctypes.c_void_p(4096)   # never dereferenced: validation fails first


def adesc(**kw):
    base = dict(B=2, HK=2, H=4, T=100, S=100, d=64, io=1, scale=0.125, left=-1, right=0)
    base.update(kw)
    return e2ttt.AttentionDesc(*[base[n] for n, _ in e2ttt.AttentionDesc._fields_])


def calls(lib, d, s=None):
    r = ctypes.byref(d)
    s = None if s is None else ctypes.byref(s)
    return (lib.e2ttt_attn_forward(r, s, *([FAKE] * 7), 1 << 50, None),
            lib.e2ttt_attn_backward(r, s, *([FAKE] * 12), 1 << 50, None))


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 2), (dict(HK=0), 2), (dict(H=3), 2), (dict(H=-4), 2), (dict(T=0), 2), (dict(S=0), 2),
    (dict(d=0), 2), (dict(scale=0.0), 2), (dict(scale=-1.0), 2), (dict(scale=math.inf), 2),
    (dict(scale=math.nan), 2), (dict(scale=3e38), 2), (dict(scale=1e-39), 2), (dict(io=2), 3), (dict(d=12), 3), (dict(d=136), 3),
    (dict(T=(1 << 29) + 1), 3), (dict(S=(1 << 29) + 1), 3), (dict(B=1 << 20, T=2048), 3),
    (dict(B=1 << 20, T=1, S=2048), 3)])
def test_bad_descriptors(lib, kw, status):
    d = adesc(**kw)
    assert calls(lib, d) == (status,) * 2
    assert lib.e2ttt_attn_scratch_bytes(ctypes.byref(d)) == 0
    assert lib.e2ttt_attn_workspace_bytes(ctypes.byref(d)) == 0


def test_null_alignment_and_sizes(lib):
    d = adesc()
    r = ctypes.byref(d)
    # forward: q k v lengths out lse workspace
    for i in (0, 1, 2, 4):
        for x, status in ((None, 1), (ctypes.c_void_p(4104), 2)):
            a = [FAKE] * 7
            a[i] = x
            assert lib.e2ttt_attn_forward(r, None, *a, 1 << 50, None) == status, i
    long = adesc(B=1, HK=1, H=1, T=64, S=8192)         # (its keys are split)
    n = lib.e2ttt_attn_workspace_bytes(ctypes.byref(long))
    assert n >= 2 * 64 * 66 * 4
    a = [FAKE] * 7
    assert lib.e2ttt_attn_forward(ctypes.byref(long), None, *a, n - 1, None) == 4
    assert lib.e2ttt_attn_forward(ctypes.byref(long), None, *a[:6], None, n, None) == 1
    assert lib.e2ttt_attn_forward(ctypes.byref(long), None, *a[:6], ctypes.c_void_p(4104), n, None) == 2
    # backward: q k v lengths out lse d_out d_lse dq dk dv scratch
    n = lib.e2ttt_attn_scratch_bytes(r)
    assert n >= 8 * 2 * 4 * 100
    for i in (0, 1, 2, 4, 5, 6, 8, 9, 10, 11):
        a = [FAKE] * 12
        a[i] = None
        assert lib.e2ttt_attn_backward(r, None, *a, n, None) == 1, i
        if i != 5:
            a[i] = ctypes.c_void_p(4104)
            assert lib.e2ttt_attn_backward(r, None, *a, n, None) == 2, i
    assert lib.e2ttt_attn_backward(r, None, *([FAKE] * 12), n - 1, None) == 4


@pytest.mark.parametrize("name,st", [
    ("q", (6400, 64, -64)), ("k", (1, 6400, 64)), ("v", (12800, 6400, (1 << 23) + 8)),
    ("out", (0, 6400, 64)), ("out", (25600, 64, 64)), ("d_out", (25600, 6400, 60)),
    ("dq", (25600, 0, 64)), ("dk", (12800, 6400, 56)), ("dv", (0, 6400, 64))])
def test_bad_strides(lib, name, st):
    d = adesc()
    s = e2ttt.AttentionStrides()
    for n in ("q", "out", "d_out", "dq"):
        setattr(s, n, e2ttt.Strides(25600, 6400, 64))
    for n in ("k", "v", "dk", "dv"):
        setattr(s, n, e2ttt.Strides(12800, 6400, 64))
    setattr(s, name, e2ttt.Strides(*st))
    f, b = calls(lib, d, s)
    if name in ("q", "k", "v", "out"):
        assert f == 2
    if name != "out" or st[2] % 8:      # (the backward reads out: elements may repeat)
        assert b == 2


def test_binding_refuses_before_the_library(lib):
    cfg = e2ttt.AttentionConfig(1, 1, 1, 4, 8)
    x = torch.zeros(1, 1, 4, 8, dtype=torch.bfloat16)
    for f in (lambda: e2ttt.attention_forward(cfg, x, x, x),
              lambda: e2ttt.attention_backward(cfg, x, x, x, x, x, x),
              lambda: e2ttt.AttentionFunction.apply(cfg, x, x, x)):
        with pytest.raises(ValueError):
            f()


def test_reference_gradients_by_differences():
    """The gradients written out in tests/attnref.py against central differences."""
    B, HK, H, T, S, d, left, right = 2, 1, 2, 6, 9, 8, 3, 1
    lengths = torch.tensor([6, 4])
    g = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x = dict(q=rn(B, H, T, d), k=rn(B, HK, S, d), v=rn(B, HK, S, d))
    d_out, d_lse = rn(B, H, T, d), rn(B, H, T)
    _, lse, ref, _ = attnref.gradients(x, 0.4, left, right, lengths, d_out, d_lse)

    def loss(y):
        o, l, a = attnref.attention(y, 0.4, left, right, lengths)
        ok = l > -math.inf
        return (o * d_out * a["live"][:, None, :, None]).sum() + (l[ok] * d_lse[ok]).sum()

    for n in x:
        for i in range(0, x[n].numel(), 7):
            e = torch.zeros(x[n].numel(), dtype=torch.float64)
            e[i] = 1e-5
            e = e.view_as(x[n])
            num = (loss(dict(x, **{n: x[n] + e})) - loss(dict(x, **{n: x[n] - e}))) / 2e-5
            assert abs(num.item() - ref[n].flatten()[i].item()) < 1e-8


def test_autograd_under_capture_is_refused(lib, monkeypatch):
    """The capture's query stands in here for a capture, and attention's calls for the
    library's: a wanted gradient is refused before anything is recorded, in either direction."""
    cfg = e2ttt.AttentionConfig(1, 1, 1, 4, 8)
    x = torch.zeros(1, 1, 4, 8, dtype=torch.bfloat16)
    on, calls = [False], []
    monkeypatch.setattr(e2ttt, "_capturing", lambda t: on[0])
    monkeypatch.setattr(e2ttt, "attention_forward", lambda cfg, q, k, v, lengths: (
        calls.append("forward"), (q + k + v, q.sum(-1).float()))[1])
    monkeypatch.setattr(e2ttt, "_attention_grads", lambda ctx, *g: (calls.append("backward"), None, x, x, x)[1:] +
                        (None,))
    for i in range(3):
        t = [x.clone().requires_grad_(n == i) for n in range(3)]
        on[0] = True
        with pytest.raises(RuntimeError, match="attention_forward and attention_backward"):
            e2ttt.AttentionFunction.apply(cfg, *t)
        assert calls == []
        with torch.no_grad():                   # no gradient is wanted: an ordinary call
            e2ttt.AttentionFunction.apply(cfg, *t)
        e2ttt.AttentionFunction.apply(cfg, *[y.detach() for y in t])
        on[0] = False
        out, _ = e2ttt.AttentionFunction.apply(cfg, *t)
        on[0] = True
        assert calls == ["forward"] * 3
        with pytest.raises(RuntimeError, match="attention_forward and attention_backward"):
            out.sum().backward()
        assert calls == ["forward"] * 3
        on[0] = False
        out, _ = e2ttt.AttentionFunction.apply(cfg, *t)
        out.sum().backward()
        assert calls == ["forward"] * 4 + ["backward"]
        calls.clear()
