"""GPU tests of attention over the 4-bit cache where its pages are split into stretches
(from 64 pages of a sequence on) and joined by a second kernel, against
tests/cacheref.py in 64 bits within the bounds derived there: every head dim, several
sequences and key heads, tiles of columns that are not full, sequences that end in the
first stretch or hold nothing, rings that wrap inside a stretch, windows, stretches
without pages, and captured calls."""
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import cacheref
from tests.test_gpu_attention import rounded, within
from tests.test_gpu_cache import IO, i32, table_of
from tests.test_gpu_delta import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def setup(B, HK, H, T, d, P, starts, lens, left, io, seed):
    """A pool whose pages hold the sequences' last tokens between whatever bytes there are."""
    g = torch.Generator().manual_seed(seed)
    n = B * P + 2
    cache = torch.randint(0, 256, (n, HK, 68 * d), generator=g, dtype=torch.uint8).cuda()
    table = table_of(B, P, n, seed)
    kv = []
    for b in range(B):                          # (sequence by sequence: they differ in length)
        end = starts[b] + lens[b]
        hold = cacheref.held(starts[b], lens[b], P)
        k, v = (torch.zeros(HK, max(end, 1), d, dtype=torch.float64) for _ in "kv")
        if len(hold):
            x = [rounded(torch.randn(1, HK, len(hold), d, generator=g, dtype=torch.float64), io) for _ in "kv"]
            fill = e2ttt.CacheConfig(1, HK, HK, len(hold), d, P, IO(io))
            e2ttt.cache_write(fill, dev(x[0], io), dev(x[1], io), cache, table[b:b + 1].to(torch.int32).cuda(),
                              i32([hold[0]]))
            for to, y in zip((k, v), x):
                to[:, hold[0]:] = cacheref.values(*cacheref.quantise(y))[0]
        kv.append((k, v))
    q = rounded(torch.randn(B, H, T, d, generator=g, dtype=torch.float64), io)
    cfg = e2ttt.CacheConfig(B, HK, H, T, d, P, IO(io), scale=d ** -0.5, left=left)
    return cfg, cache, table.to(torch.int32).cuda(), kv, q


def dirty(cfg):
    n = e2ttt.cache_workspace_bytes(cfg)
    assert n > 256                              # (it is split)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


SPLIT = [  # B, HK, H, T, d, P, starts, lengths, left
    (3, 2, 6, 3, 32, 70, [4400, 10, 0], [3, 1, 0], -1),     # 9 columns; short and dead sequences
    (2, 1, 5, 4, 64, 66, [9000, 4300], [4, 4], -1),         # 20 columns; a ring that wraps twice
    (1, 3, 3, 1, 96, 80, [5100], [1], 4990),
    (6, 1, 2, 2, 64, 64, [4090, 64, 4000, 0, 100, 2000], [2, 2, 1, 2, 0, 2], -1),
    (2, 2, 4, 5, 128, 130, [12000, 8300], [5, 2], 4500),    # a ring and a window
    (1, 1, 17, 1, 32, 200, [12799], [1], -1),
    (1, 2, 2, 1, 96, 90, [63], [1], -1)]                    # one page: every other stretch is empty


@pytest.mark.parametrize("c", SPLIT)
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_split_attention(c, io):
    B, HK, H, T, d, P, starts, lens, left = c
    print("split", c, io, flush=True)
    cfg, cache, table, kv, q = setup(*c, io, d + T)
    out, lse, bounds = cacheref.attend(q, kv, starts, lens, P, left, d ** -0.5)
    qd = dev(q, io, "bthd").clone(memory_format=torch.preserve_format)
    for b in range(B):
        qd[b, :, lens[b]:] = math.nan
    l = torch.full((B, H, T), math.nan, device="cuda")
    o, _ = e2ttt.cache_attention(cfg, qd, cache, table, i32(starts), i32(lens), lse=l, workspace=dirty(cfg))
    bo, bl = bounds(io == "bf16")
    within("out", o, out, bo, 2.0 ** -8 if io == "bf16" else 2.0 ** -18)
    within("lse", l, lse, bl, 2.0 ** -18)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_stretches_without_pages(io):
    """Sequences with a stretch of entries that are no page, with only one page left, and with none."""
    B, HK, H, T, d, P = 3, 2, 4, 2, 64, 70
    starts, lens = [4470, 4460, 4450], [2, 2, 2]
    cfg, cache, table, kv, q = setup(B, HK, H, T, d, P, starts, lens, -1, io, 5)
    gone = {(0, i) for i in range(13, 43)} | {(1, i) for i in range(70) if i != 30} | {(2, i) for i in range(70)}
    for b, i in gone:
        table[b, i] = -1
    out, lse, bounds = cacheref.attend(q, kv, starts, lens, P, -1, d ** -0.5, gone)
    l = torch.full((B, H, T), math.nan, device="cuda")
    o, _ = e2ttt.cache_attention(cfg, dev(q, io), cache, table, i32(starts), i32(lens), lse=l, workspace=dirty(cfg))
    assert (o[2] == 0).all() and (l[2] == -math.inf).all()
    bo, bl = bounds(io == "bf16")
    within("out", o, out, bo, 2.0 ** -8 if io == "bf16" else 2.0 ** -18)
    within("lse", l, lse, bl, 2.0 ** -18)


def test_split_calls_as_graphs_on_two_streams():
    """Two captured split calls with workspaces of their own, replayed at once."""
    runs = []
    for seed, d in ((1, 64), (2, 96)):
        c = (2, 2, 6, 3, d, 100, [6300, 2000], [3, 3], -1)
        cfg, cache, table, _, q = setup(*c, "bf16", seed)
        x, at, ws = dev(q, "bf16"), i32(c[6]), dirty(cfg)
        lse, ref_lse = (torch.zeros(2, 6, 3, device="cuda") for _ in "ab")
        ref, _ = e2ttt.cache_attention(cfg, x, cache, table, at, lse=ref_lse)
        out = torch.empty_like(ref)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            e2ttt.cache_attention(cfg, x, cache, table, at, out=out, lse=lse, workspace=ws)
        runs.append((graph, torch.cuda.Stream(), ref, ref_lse, out, lse, (cache, table, x, at, ws)))
    for _ in range(4):
        for r in runs:
            r[4].zero_()
            r[5].zero_()
        torch.cuda.synchronize()
        for r in runs:
            with torch.cuda.stream(r[1]):
                r[0].replay()
        torch.cuda.synchronize()
        for _, _, ref, ref_lse, out, lse, _ in runs:
            assert torch.equal(out, ref) and torch.equal(lse, ref_lse)
