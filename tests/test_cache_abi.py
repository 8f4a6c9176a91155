"""Refusals and sizes of the 4-bit cache's entry points, and the reference that the
GPU tests compare with; no call here reaches a kernel."""
import ctypes
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import cacheref


@pytest.fixture(scope="module")
def lib():
    return e2ttt.load()


FAKE = ctypes.c_void_p(4096)   # never dereferenced: validation fails first


def cdesc(**kw):
    base = dict(B=2, HK=2, H=4, T=3, d=64, pages=10, io=1, scale=0.125, left=-1)
    base.update(kw)
    return e2ttt.CacheDesc(*[base[n] for n, _ in e2ttt.CacheDesc._fields_])


def calls(lib, d, s=None, n=8):
    r = ctypes.byref(d)
    s = None if s is None else ctypes.byref(s)
    return (lib.e2ttt_cache_write(r, s, *([FAKE] * 6), n, None),
            lib.e2ttt_cache_read(r, s, *([FAKE] * 4), n, FAKE, FAKE, None),
            lib.e2ttt_cache_attend(r, s, *([FAKE] * 5), n, FAKE, FAKE, FAKE, 1 << 50, None))


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), 2), (dict(HK=0), 2), (dict(T=0), 2), (dict(d=0), 2), (dict(pages=0), 2), (dict(io=2), 3),
    (dict(d=48), 3), (dict(d=16), 3), (dict(d=160), 3), (dict(T=(1 << 29) + 1), 3),
    (dict(pages=(1 << 25) + 1), 3), (dict(B=1 << 20, HK=1 << 10, H=1 << 10), 3),
    (dict(B=1 << 16, HK=16, H=16, T=4096), 3)])
def test_bad_descriptors(lib, kw, status):
    d = cdesc(**kw)
    assert calls(lib, d) == (status,) * 3
    assert lib.e2ttt_cache_workspace_bytes(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw,status", [(dict(H=3), 2), (dict(H=0), 2), (dict(scale=0.0), 2),
                                       (dict(scale=math.nan), 2), (dict(scale=math.inf), 2),
                                       (dict(B=1 << 20, HK=4, H=64, T=16), 3)])
def test_bad_descriptors_of_attention(lib, kw, status):
    d = cdesc(**kw)
    assert calls(lib, d)[2] == status
    assert lib.e2ttt_cache_workspace_bytes(ctypes.byref(d)) == 0


def test_null_alignment_and_sizes(lib):
    d = cdesc()
    r = ctypes.byref(d)
    odd = ctypes.c_void_p(4104)
    # write: k v starts lengths table cache
    for i in (0, 1, 4, 5):
        a = [FAKE] * 6
        a[i] = None
        assert lib.e2ttt_cache_write(r, None, *a, 8, None) == 1, i
        if i != 4:
            a[i] = odd
            assert lib.e2ttt_cache_write(r, None, *a, 8, None) == 2, i
    # read: starts lengths table cache | k v
    for i in (2, 3, 4, 5):
        a = [FAKE] * 6
        a[i] = None
        assert lib.e2ttt_cache_read(r, None, *a[:4], 8, *a[4:], None) == 1, i
        if i != 2:
            a[i] = odd
            assert lib.e2ttt_cache_read(r, None, *a[:4], 8, *a[4:], None) == 2, i
    # attend: q starts lengths table cache | out lse workspace
    n = lib.e2ttt_cache_workspace_bytes(r)
    for i in (0, 3, 4, 5, 7):
        a = [FAKE] * 8
        a[i] = None
        assert lib.e2ttt_cache_attend(r, None, *a[:5], 8, *a[5:], n, None) == 1, i
        if i != 3:
            a[i] = odd
            assert lib.e2ttt_cache_attend(r, None, *a[:5], 8, *a[5:], n, None) == 2, i
    assert lib.e2ttt_cache_attend(r, None, *([FAKE] * 5), 8, FAKE, FAKE, FAKE, n - 1, None) == 4
    assert calls(lib, d, n=0) == (2,) * 3 and calls(lib, d, n=-4) == (2,) * 3


def test_the_largest_launch(lib):
    """2^32 threads are too many for a launch; a workgroup that attends has 512."""
    at = lambda B: e2ttt.cache_workspace_bytes(e2ttt.CacheConfig(B, 1, 1, 1, 32, 1))
    assert at((1 << 23) - 1) > 0 and at(1 << 23) == 0


def test_sizes(lib):
    assert e2ttt.cache_page_bytes(3, 96) == 3 * 68 * 96
    assert e2ttt.cache_page_bytes(0, 64) == e2ttt.cache_page_bytes(2, 40) == e2ttt.cache_page_bytes(2, 256) == 0
    assert e2ttt.cache_workspace_bytes(e2ttt.CacheConfig(1, 1, 1, 1, 64, 1)) > 0


@pytest.mark.parametrize("name,st", [("q", (768, 192, -64)), ("k", (384, 192, 60)), ("v", (1, 192, 64)),
                                     ("out", (0, 192, 64))])
def test_bad_strides(lib, name, st):
    s = e2ttt.CacheStrides()
    for n, h in (("q", 4), ("out", 4), ("k", 2), ("v", 2)):
        setattr(s, n, e2ttt.Strides(192 * h, 192, 64))
    setattr(s, name, e2ttt.Strides(*st))
    w, r, a = calls(lib, cdesc(), s)
    assert (a if name in ("q", "out") else w) == 2
    assert name in ("q", "out") or r == 2


def test_read_refuses_rows_that_overlap(lib):
    s = e2ttt.CacheStrides()
    for n in ("k", "v"):
        setattr(s, n, e2ttt.Strides(384, 0, 64))
    assert calls(lib, cdesc(), s)[1] == 2


def test_binding_refuses_before_the_library(lib):
    cfg = e2ttt.CacheConfig(1, 1, 1, 1, 64, 2)
    x = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    cache, table = torch.zeros(3, 1, 68 * 64, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    for f in (lambda: e2ttt.cache_write(cfg, x, x, cache, table),
              lambda: e2ttt.cache_read(cfg, cache, table),
              lambda: e2ttt.cache_attention(cfg, x, cache, table)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(e2ttt.E2TTTError):
        e2ttt.alloc_cache(e2ttt.CacheConfig(1, 1, 1, 1, 48, 2), 3, device="cpu")


def test_reference_values():
    """The sixteen values, the scale's border at 7 and the ties, by hand."""
    x = torch.zeros(2, 32, dtype=torch.float64)
    x[0, :9] = torch.tensor([7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.5])
    x[1, :3] = torch.tensor([7.5, 0.5, -1.5])
    code, exp = cacheref.quantise(x)
    assert exp.flatten().tolist() == [127, 128]
    assert cacheref.values(code, exp)[0, :9].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -6.0]
    assert cacheref.values(code, exp)[1, :3].tolist() == [8.0, 0.0, -2.0]
