"""Refusals and sizes of the delta and query/key entry points, and the rotary
frequencies; no call here reaches a kernel."""
import ctypes
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt


@pytest.fixture(scope="module")
def lib():
    return e2ttt.load()


FAKE = ctypes.c_void_p(4096)   # never dereferenced: validation fails first


def ddesc(**kw):
    base = dict(B=2, HK=2, H=4, T=100, dk=64, dv=64, io=1, scale=1.0)
    base.update(kw)
    return e2ttt.DeltaDesc(*[base[n] for n, _ in e2ttt.DeltaDesc._fields_])


def calls(lib, d, s=None):
    r = ctypes.byref(d)
    s = None if s is None else ctypes.byref(s)
    return (lib.e2ttt_delta_forward(r, s, *([FAKE] * 10), 1 << 50, 0, None),
            lib.e2ttt_delta_backward(r, s, *([FAKE] * 7), 1 << 50, *([FAKE] * 9), 1 << 50, None),
            lib.e2ttt_delta_step(r, s, *([FAKE] * 7), 8, FAKE, None))


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 2), (dict(HK=0), 2), (dict(H=3), 2), (dict(H=0), 2), (dict(T=0), 2), (dict(T=-5), 2),
    (dict(dk=0), 2), (dict(dv=-8), 2), (dict(scale=math.inf), 2), (dict(scale=math.nan), 2),
    (dict(io=2), 3), (dict(dk=12), 3), (dict(dk=136), 3), (dict(dv=20), 3), (dict(dv=264), 3),
    (dict(B=1 << 14, HK=1 << 10, H=1 << 10), 3), (dict(B=1 << 12, HK=8, H=8, T=1 << 21), 3)])
def test_bad_descriptors(lib, kw, status):
    d = ddesc(**kw)
    assert calls(lib, d) == (status,) * 3
    assert lib.e2ttt_delta_workspace_bytes(ctypes.byref(d), 1) == 0
    assert lib.e2ttt_delta_scratch_bytes(ctypes.byref(d)) == 0


def test_null_alignment_and_sizes(lib):
    d = ddesc()
    r = ctypes.byref(d)
    big = 1 << 50
    # forward: q k v eta log_gamma lengths w_in out w_out workspace
    for i in (0, 1, 2, 3, 7, 9):
        a = [FAKE] * 10
        a[i] = None
        assert lib.e2ttt_delta_forward(r, None, *a, big, 0, None) == 1, i
    for i in (0, 1, 2, 6, 7, 8, 9):
        a = [FAKE] * 10
        a[i] = ctypes.c_void_p(4104)
        assert lib.e2ttt_delta_forward(r, None, *a, big, 0, None) == 2, i
    for save in (0, 1):
        n = lib.e2ttt_delta_workspace_bytes(r, save)
        assert lib.e2ttt_delta_forward(r, None, *([FAKE] * 10), n - 1, save, None) == 4
    assert lib.e2ttt_delta_forward(r, None, *([FAKE] * 10), lib.e2ttt_delta_workspace_bytes(r, 0), 1, None) == 4
    # backward: q k v eta log_gamma lengths workspace | d_out d_w_out dq dk dv d_eta d_log_gamma d_w_in scratch
    def back(i=None, x=None, ws=big, sc=big):
        a = [FAKE] * 16
        if i is not None:
            a[i] = x
        return lib.e2ttt_delta_backward(r, None, *a[:7], ws, *a[7:], sc, None)
    for i in (0, 1, 2, 3, 4, 6, 7, 9, 10, 11, 12, 13, 15):    # log_gamma, d_log_gamma: both or neither
        assert back(i, None) == 1, i
    for i in (0, 1, 2, 6, 7, 8, 9, 10, 11, 14, 15):
        assert back(i, ctypes.c_void_p(4100)) == 2, i
    assert back(ws=lib.e2ttt_delta_workspace_bytes(r, 1) - 1) == 4
    assert back(sc=lib.e2ttt_delta_scratch_bytes(r) - 1) == 4
    # step: q k v eta log_gamma w slots, n_slots, out
    for i in (0, 1, 2, 3, 5):
        a = [FAKE] * 7
        a[i] = None
        assert lib.e2ttt_delta_step(r, None, *a, 8, FAKE, None) == 1, i
    assert lib.e2ttt_delta_step(r, None, *([FAKE] * 7), 8, None, None) == 1
    assert lib.e2ttt_delta_step(r, None, *([FAKE] * 7), 0, FAKE, None) == 2
    assert lib.e2ttt_delta_step(r, None, *([FAKE] * 6), None, 1, FAKE, None) == 2   # fewer states than rows
    for i in (0, 1, 2, 5):
        a = [FAKE] * 7
        a[i] = ctypes.c_void_p(4100)
        assert lib.e2ttt_delta_step(r, None, *a, 8, FAKE, None) == 2, i


def test_workspace_without_saving_is_bounded(lib):
    short = ddesc(B=1, HK=16, H=16, T=64, dk=128, dv=128)
    for kw in (dict(B=1, HK=16, H=16), dict(B=1, HK=1, H=1), dict(B=16, HK=16, H=16),
               dict(B=1, HK=1, H=2, dv=32)):
        long = ddesc(**dict(dict(T=1 << 20, dk=128, dv=128), **kw))
        state = long.B * long.H * long.dk * long.dv * 4
        assert lib.e2ttt_delta_workspace_bytes(ctypes.byref(long), 0) <= (704 << 20) + state, kw
    assert lib.e2ttt_delta_workspace_bytes(ctypes.byref(short), 0) < 1 << 20
    # saving: a state and an update per chunk and unit
    assert lib.e2ttt_delta_workspace_bytes(ctypes.byref(short), 1) >= 16 * (128 * 128 + 128 * 64) * 4


def strides(**kw):
    """C order of ddesc() but for the tensors given."""
    s = e2ttt.DeltaStrides()
    for n, _ in e2ttt.DeltaStrides._fields_:
        heads = 2 if n in ("q", "k", "dq", "dk") else 4
        inner = 1 if "eta" in n or "gamma" in n else 64
        setattr(s, n, e2ttt.Strides(heads * 100 * inner, 100 * inner, inner))
    for n, v in kw.items():
        setattr(s, n, e2ttt.Strides(*v))
    return s


@pytest.mark.parametrize("name,st,which", [
    ("q", (12800, 6400, -64), (0, 1, 2)), ("k", (12800, 6400, 1 << 50), (0, 1, 2)),
    ("v", (25600, 6400, 68), (0, 1, 2)), ("eta", (400, -100, 1), (0, 1, 2)),
    ("out", (25600, 6400, 0), (0, 2)), ("out", (25600, 6400, 56), (0, 2)),
    ("out", (25600, 64, 64), (0, 2)), ("d_out", (25600, 6400, 12), (1,)),
    ("dq", (12800, 0, 64), (1,)), ("dk", (0, 6400, 64), (1,)), ("dv", (25600, 6400, 32), (1,)),
    ("d_eta", (400, 100, 0), (1,)), ("d_log_gamma", (100, 100, 1), (1,))])
def test_bad_strides(lib, name, st, which):
    got = calls(lib, ddesc(), strides(**{name: st}))
    for i in which:
        assert got[i] == 2, (name, st, i)


def qdesc(**kw):
    base = dict(B=2, H=4, HK=2, T=100, d=64, rot=64, io=1, flags=3, eps=1e-6, rot_scale=1.0)
    base.update(kw)
    return e2ttt.QKDesc(*[base[n] for n, _ in e2ttt.QKDesc._fields_])


def qcalls(lib, d):
    r = ctypes.byref(d)
    return (lib.e2ttt_qk_forward(r, None, *([FAKE] * 6), None),
            lib.e2ttt_qk_backward(r, None, *([FAKE] * 8), None))


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 2), (dict(H=0), 2), (dict(HK=-1), 2), (dict(T=0), 2), (dict(d=0), 2), (dict(rot=-2), 2),
    (dict(rot=66), 2), (dict(rot=3), 2), (dict(eps=0.0), 2), (dict(eps=math.nan), 2),
    (dict(rot_scale=math.inf), 2), (dict(io=5), 3), (dict(flags=8), 3), (dict(d=68), 3),
    (dict(d=264), 3), (dict(B=1 << 20, T=1 << 10), 3)])
def test_qk_bad_descriptors(lib, kw, status):
    assert qcalls(lib, qdesc(**kw)) == (status,) * 2


def test_qk_null_and_alignment(lib):
    r = ctypes.byref(qdesc())
    # forward: q k inv_freq positions q_out k_out; backward: q k inv_freq positions d_q d_k dq dk
    for i in (0, 1, 2, 4, 5):
        a = [FAKE] * 6
        a[i] = None
        assert lib.e2ttt_qk_forward(r, None, *a, None) == 1, i
    for i in (0, 1, 4, 5):
        a = [FAKE] * 6
        a[i] = ctypes.c_void_p(4104)
        assert lib.e2ttt_qk_forward(r, None, *a, None) == 2, i
    for i in (0, 1, 2, 4, 5, 6, 7):
        a = [FAKE] * 8
        a[i] = None
        assert lib.e2ttt_qk_backward(r, None, *a, None) == 1, i
    for i in (0, 1, 4, 5, 6, 7):
        a = [FAKE] * 8
        a[i] = ctypes.c_void_p(4104)
        assert lib.e2ttt_qk_backward(r, None, *a, None) == 2, i
    assert lib.e2ttt_qk_forward(None, None, *([FAKE] * 6), None) == 1


def test_binding_refuses_what_is_not_on_the_gpu():
    cfg = e2ttt.DeltaConfig(1, 1, 1, 4, 16, 16)
    x = torch.zeros(1, 1, 4, 16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        e2ttt.delta_forward(cfg, x, x, x, torch.zeros(1, 1, 4))
    with pytest.raises(ValueError):
        e2ttt.delta_step(cfg, x, x, x, torch.zeros(1, 1, 4), None, torch.zeros(1, 1, 16, 16))
    with pytest.raises(ValueError):
        e2ttt.qk_forward(e2ttt.QKConfig(1, 1, 1, 4, 16, 16), x, x, torch.zeros(8))


def test_rotary_frequencies():
    f, m = e2ttt.rotary_frequencies(64, device="cpu")
    i = torch.arange(32, dtype=torch.float64)
    assert m == 1.0 and torch.equal(f, (10000.0 ** (-2 * i / 64)).float())
    g, m = e2ttt.rotary_frequencies(64, factor=4.0, device="cpu")
    assert m == 1.0 and torch.allclose(g, f / 4, rtol=1e-6)
    h, m = e2ttt.rotary_frequencies(64, factor=4.0, original=4096, device="cpu")
    assert abs(m - (0.1 * math.log(4.0) + 1.0)) < 1e-12
    turns = 4096 * f.double() / (2 * math.pi)
    kept, slow = turns > 40, turns < 0.8
    assert kept.any() and slow.any()
    assert torch.allclose(h[kept], f[kept], rtol=1e-6) and torch.allclose(h[slow], f[slow] / 4, rtol=1e-6)
    assert ((h <= f) & (h >= f / 4 * 0.999999)).all() and (h[1:] <= h[:-1]).all()
    assert e2ttt.rotary_frequencies(0, device="cpu")[0].numel() == 0
    for bad in (dict(rot=3), dict(rot=64, base=0.5), dict(rot=64, factor=0.5),
                dict(rot=64, factor=2.0, original=-1)):
        with pytest.raises(ValueError):
            e2ttt.rotary_frequencies(device="cpu", **bad)


def test_launches_of_more_than_32_bits_of_threads(lib):
    def size(save, **kw):
        return lib.e2ttt_delta_workspace_bytes(ctypes.byref(ddesc(**kw)), save)

    assert size(0, B=1 << 21, HK=1, H=1, dv=64) > 0
    assert size(0, B=1 << 21, HK=1, H=1, dv=256) == 0
    big = dict(B=1, HK=1024, H=1024, T=1 << 20)
    assert size(0, **big) > 0 and size(1, **big) == 0
    assert lib.e2ttt_delta_scratch_bytes(ctypes.byref(ddesc(**big))) == 0
    assert calls(lib, ddesc(**big))[1] == 3
    assert qcalls(lib, qdesc(B=1 << 14, T=1 << 14, H=1, HK=0, rot=2)) == (3, 3)


def test_segments_by_their_first_pass(lib):
    """The pass that segments cost beside the chain is as wide as values and keys together:
    short chains of many units run without them (no room is asked for the segments' states),
    heads of 128 sooner than those of 64."""
    def each(B, T, d):
        return lib.e2ttt_delta_workspace_bytes(ctypes.byref(ddesc(B=B, HK=1, H=1, T=T, dk=d, dv=d)), 0) / B

    plain = each(96, 1088, 128)
    assert abs(each(80, 1088, 128) - plain) < 1024 and abs(each(48, 1088, 128) - plain) < 1024
    assert each(32, 1088, 128) > plain + (1 << 18) and each(64, 8192, 128) > each(96, 8192, 128) + (1 << 18)
    plain = each(96, 1088, 64)
    assert abs(each(80, 1088, 64) - plain) < 1024 and each(64, 1088, 64) > plain + (1 << 16)
    assert abs(each(80, 512, 64) - each(96, 512, 64)) < 1024 and each(80, 2048, 64) > each(96, 2048, 64) + (1 << 16)


@pytest.mark.parametrize("kw,rows", [
    (dict(H=1, HK=0, d=128, rot=128, io=1), 1 << 29), (dict(H=1, HK=0, d=64, rot=64, io=0), 1 << 29),
    (dict(H=1, HK=0, d=256, rot=256, io=1), 1 << 28), (dict(H=2, HK=1, d=256, rot=6, io=1), 1 << 26),
    (dict(H=1, HK=0, d=16, rot=2, io=1), 1 << 29)])
def test_qk_lanes_of_a_launch(lib, kw, rows):
    """The documented limit of rows times lanes, from both sides (a null pointer, looked at
    behind the descriptor, ends the calls below it)."""
    h = kw["rot"] // 2
    v = next(v for v in ((8,) if kw["io"] else ()) + (4, 2, 1) if h % v == 0)
    lanes = 1
    while lanes < min(64, -(-kw["d"] // (2 * v))):
        lanes *= 2
    assert rows * lanes * -(-(kw["H"] + kw["HK"]) // 8) == 1 << 32
    assert qcalls(lib, qdesc(B=1 << 10, T=rows >> 10, **kw)) == (3, 3)
    below = ctypes.byref(qdesc(B=1, T=rows - 256 // lanes, **kw))
    assert lib.e2ttt_qk_forward(below, None, *([None] * 6), None) == 1
    assert lib.e2ttt_qk_backward(below, None, *([None] * 8), None) == 1


def test_qk_eps_is_a_normal_number(lib):
    """A subnormal eps gave NaN for a row of zeros."""
    assert qcalls(lib, qdesc(eps=1e-40)) == (2, 2) and qcalls(lib, qdesc(eps=-1.0)) == (2, 2)
    r = ctypes.byref(qdesc(eps=2.0 ** -126))
    assert lib.e2ttt_qk_forward(r, None, *([None] * 6), None) == 1
    assert lib.e2ttt_qk_forward(ctypes.byref(qdesc(eps=1e-40, flags=1)), None, *([None] * 6), None) == 1
