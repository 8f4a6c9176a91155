"""GPU tests of the 4-bit cache: written pages byte by byte against
tests/cacheref.py (nothing else changes), what is read back exactly, and attention
over it in 64 bits within the bounds derived there."""
import math

import pytest
import torch

from paper_2608_21308_amd import e2ttt
from tests import cacheref
from tests.test_gpu_attention import rounded, within
from tests.test_gpu_delta import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    e2ttt.load()


def IO(io):
    return e2ttt.DT_BF16 if io == "bf16" else e2ttt.DT_F32


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32).cuda()


def rows(B, HK, T, d, io, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, B, HK, T, d, generator=g, dtype=torch.float64)
    x = x * torch.exp2(torch.randint(-20, 20, (2, B, HK, T, 1), generator=g))
    return [rounded(y, io) for y in x]


def table_of(B, P, n, seed=0):
    return torch.randperm(n, generator=torch.Generator().manual_seed(seed))[:B * P].view(B, P)


def writes(want, table, k, v, starts, lengths, P):
    """The same into a host pool [n, HK, 68 d]."""
    (kc, ke), (vc, ve) = cacheref.quantise(k), cacheref.quantise(v)
    B, HK = k.shape[:2]
    for b in range(B):
        hold = cacheref.held(starts[b], lengths[b], P)
        for t in range(lengths[b]):
            p = starts[b] + t
            page = int(table[b, p // 64 % P]) if p >= 0 else -1
            if p in hold and 0 <= page < want.shape[0]:
                for h in range(HK):
                    cacheref.put(want[page, h], p % 64, kc[b, h, t], ke[b, h, t], vc[b, h, t], ve[b, h, t])


CASES = [  # B, HK, T, d, P, starts, lengths
    (1, 1, 1, 32, 1, [0], None), (2, 3, 1, 64, 3, [63, 130], None), (2, 1, 5, 96, 2, [62, 0], [5, 3]),
    (3, 2, 70, 128, 3, [0, 61, 130], [70, 0, 33]), (2, 1, 200, 64, 2, [7, 1], [200, 150]),
    (1, 2, 6, 32, 2, [3], None), (2, 1, 9, 64, 4, [-4, -20], None), (1, 1, 130, 32, 1, [0], None),
    (2, 1, 7, 64, 3, [2 ** 31 - 70, 2 ** 30], [7, 99])]


@pytest.mark.parametrize("c", CASES)
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_write_and_read(c, io):
    B, HK, T, d, P, starts, lengths = c
    print("cache", c, io, flush=True)
    n, lens = B * P + 2, [T] * B if lengths is None else [max(0, min(T, x)) for x in lengths]
    k, v = rows(B, HK, T, d, io, T + d)
    table = table_of(B, P, n)
    g = torch.Generator().manual_seed(9)
    pool = torch.randint(0, 254, (n, HK, 68 * d), generator=g, dtype=torch.uint8)
    cache, want = pool.clone().cuda(), pool.clone()
    writes(want, table, k, v, starts, lens, P)
    cfg = e2ttt.CacheConfig(B, HK, HK, T, d, P, IO(io))
    layout = "bthd" if T % 2 else "bhtd"
    args = (table.to(torch.int32).cuda(), i32(starts), i32(lengths))
    e2ttt.cache_write(cfg, dev(k, io, layout), dev(v, io, layout), cache, *args)
    assert torch.equal(cache.cpu(), want)
    gk, gv = e2ttt.cache_read(cfg, cache, *args)
    for got, x in ((gk, k), (gv, v)):
        ref = cacheref.values(*cacheref.quantise(x))
        for b in range(B):
            hold = cacheref.held(starts[b], lens[b], P)
            for t in range(T):
                if t >= lens[b] or starts[b] + t not in hold:
                    ref[b, :, t] = 0.0
        assert torch.equal(got.double().cpu(), ref)
    # into views of another order, where nothing else is written
    wide = torch.full((B, T, 2 * HK, d), 7.0, dtype=gk.dtype, device="cuda")
    out = (wide[:, :, :HK].transpose(1, 2), wide[:, :, HK:].transpose(1, 2))
    e2ttt.cache_read(cfg, cache, *args, out=out)
    assert torch.equal(out[0], gk) and torch.equal(out[1], gv)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_borders_and_non_finite(io):
    """Ties between codes, the largest and the smallest scales, zeros of both signs, and
    blocks with an infinity or NaN."""
    d, T = 128, 12
    k = torch.zeros(1, 1, T, d, dtype=torch.float64)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, -0.0, -0.25, -7.0, 0.125])
    for t, e in enumerate([0, -3, 40, 118, -118]):
        k[0, 0, t, :14] = ties * 2.0 ** e
        k[0, 0, t, 40] = 7.0625 * 2.0 ** e           # above 7: the next power
        k[0, 0, t, 41] = 0.5 * 2.0 ** e
        k[0, 0, t, 64] = 2.0 ** -126                 # below the least scale's steps
        k[0, 0, t, 96] = 2.0 ** 126
    k[0, 0, 6, 3], k[0, 0, 7, 33], k[0, 0, 8, 65] = math.nan, math.inf, -math.inf
    k = rounded(k, io)
    cfg = e2ttt.CacheConfig(1, 1, 1, T, d, 1, IO(io))
    cache = e2ttt.alloc_cache(cfg, 1)
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    e2ttt.cache_write(cfg, dev(k, io), dev(k.flip(2), io), cache, table)
    gk, gv = e2ttt.cache_read(cfg, cache, table)
    ref = cacheref.values(*cacheref.quantise(k))
    assert torch.isnan(ref).sum() == 3 * 32
    assert torch.equal(torch.nan_to_num(gk.double().cpu(), nan=1e300), torch.nan_to_num(ref, nan=1e300))
    assert torch.equal(torch.nan_to_num(gv.double().cpu(), nan=1e300),
                       torch.nan_to_num(ref.flip(2), nan=1e300))


ATTEND = [  # B, HK, H, T, d, P, starts, lengths, left
    (1, 1, 1, 1, 32, 1, [0], None, -1), (2, 2, 2, 1, 64, 5, [200, 63], None, -1),
    (2, 1, 4, 3, 128, 9, [500, 64], [3, 0], 130), (3, 2, 6, 5, 96, 4, [180, 251, 3], [5, 4, 1], -1),
    (2, 1, 8, 8, 64, 40, [2300, 700], None, 2000), (1, 1, 3, 2, 64, 3, [1000], None, 100),
    (1, 2, 4, 1, 128, 30, [1900], None, 0), (2, 1, 1, 4, 32, 6, [-2, -9], None, -1),
    (1, 1, 5, 70, 64, 4, [100], None, 50), (1, 1, 16, 2, 128, 70, [4400], None, -1),
    (1, 1, 2, 3, 64, 2, [2 ** 31 - 80], None, 20)]


@pytest.mark.parametrize("c", ATTEND)
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_attention(c, io):
    B, HK, H, T, d, P, starts, lengths, left = c
    print("attend", c, io, flush=True)
    lens = [T] * B if lengths is None else lengths
    n = B * P + 2
    g = torch.Generator().manual_seed(d + T)
    table = table_of(B, P, n, 3)
    cfg1 = e2ttt.CacheConfig(B, HK, H, T, d, P, IO(io), scale=d ** -0.5, left=left)
    # pages start as whatever bytes there are, NaN scales among them
    cache = torch.randint(0, 256, (n, HK, 68 * d), generator=g, dtype=torch.uint8).cuda()
    kv, ends = [], [s + x for s, x in zip(starts, lens)]
    far = max(0, min(ends) - 64 * P - 200) // 64 * 64      # (positions before this are gone)
    most = max(1, max(ends) - far)
    k, v = (torch.randn(B, HK, most, d, generator=g, dtype=torch.float64) for _ in "kv")
    k, v = rounded(k, io), rounded(v, io)
    tb = table.to(torch.int32).cuda()
    fill = e2ttt.CacheConfig(B, HK, H, most, d, P, IO(io))
    held = [max(0, e - far) for e in ends]
    e2ttt.cache_write(fill, dev(k, io), dev(v, io), cache, tb, i32([far] * B), i32(held))
    k, v = (cacheref.values(*cacheref.quantise(x)) for x in (k, v))
    for b in range(B):
        kv.append((k[b], v[b]))
    q = rounded(torch.randn(B, H, T, d, generator=g, dtype=torch.float64), io)
    out, lse, bounds = cacheref.attend(q, kv, [s - far for s in starts], lens, P, left, d ** -0.5)
    qd = dev(q, io, "bthd" if T > 1 else "bhtd").clone(memory_format=torch.preserve_format)
    for b in range(B):
        qd[b, :, lens[b]:] = math.nan
    l = torch.full((B, H, T), math.nan, device="cuda")
    o, _ = e2ttt.cache_attention(cfg1, qd, cache, tb, i32(starts), i32(lengths), lse=l)
    bo, bl = bounds(io == "bf16")
    within("out", o, out, bo, 2.0 ** -8 if io == "bf16" else 2.0 ** -18)
    within("lse", l, lse, bl, 2.0 ** -18)


def small(io="bf16", B=3, HK=2, H=4, d=64, P=6, n=30, held=300, seed=0, T=1, left=-1):
    g = torch.Generator().manual_seed(seed)
    cfg = e2ttt.CacheConfig(B, HK, H, T, d, P, IO(io), scale=d ** -0.5, left=left)
    fill = e2ttt.CacheConfig(B, HK, H, held, d, P, IO(io))
    cache, table = e2ttt.alloc_cache(cfg, n), table_of(B, P, n, seed).to(torch.int32).cuda()
    k, v = (rounded(torch.randn(B, HK, held, d, generator=g, dtype=torch.float64), io) for _ in "kv")
    e2ttt.cache_write(fill, dev(k, io), dev(v, io), cache, table)
    q = rounded(torch.randn(B, H, T, d, generator=g, dtype=torch.float64), io)
    return cfg, cache, table, k, v, q


def test_pages_that_are_none():
    """Entries outside the pool: nothing is written there, zeros are read, and
    attention goes on without them."""
    cfg, cache, table, k, v, q = small(held=300)
    table[0, 1], table[1, 0], table[2] = -1, 30, torch.iinfo(torch.int32).min
    before = cache.clone()
    fill = e2ttt.CacheConfig(3, 2, 4, 300, 64, 6)
    e2ttt.cache_write(fill, dev(-k, "bf16"), dev(v, "bf16"), cache, table)
    same = [i for i in range(30) if not (table == i).any()]
    assert torch.equal(cache[same], before[same])
    gk, _ = e2ttt.cache_read(fill, cache, table)
    ref = cacheref.values(*cacheref.quantise(-k))
    ref[0, :, 64:128], ref[1, :, :64], ref[2] = 0.0, 0.0, 0.0
    assert torch.equal(gk.double().cpu(), ref)
    k, v = (cacheref.values(*cacheref.quantise(x)) for x in (-k, v))
    gone = {(0, 1), (1, 0)} | {(2, i) for i in range(6)}
    out, lse, bounds = cacheref.attend(q, list(zip(k, v)), [299] * 3, [1] * 3, 6, -1, 0.125, gone)
    l = torch.empty(3, 4, 1, device="cuda")
    o, _ = e2ttt.cache_attention(cfg, dev(q, "bf16"), cache, table, i32([299] * 3), lse=l)
    assert not o[2].any() and torch.isinf(l[2]).all()
    bo, bl = bounds(True)
    within("out", o, out, bo, 2.0 ** -8)
    within("lse", l, lse, bl, 2.0 ** -18)


def test_zeros_beside_nan():
    """A token whose page is none and that sees no other is zero also where the call's
    other token reads a NaN."""
    for io in ("bf16", "f32"):
        cfg = e2ttt.CacheConfig(1, 1, 2, 2, 64, 2, IO(io), left=0)
        k, v = (dev(x, io) for x in rows(1, 1, 2, 64, io, 5))
        v[0, 0, 0, 3] = math.nan
        cache, table, starts = e2ttt.alloc_cache(cfg, 2), i32([[1, -1]]), i32([63])
        e2ttt.cache_write(cfg, k, v, cache, table, starts)
        lse = torch.zeros(1, 2, 2, device="cuda")
        q = dev(rows(1, 2, 2, 64, io, 6)[0], io)
        out, _ = e2ttt.cache_attention(cfg, q, cache, table, starts, lse=lse)
        assert torch.isnan(out[0, :, 0, :32]).all() and torch.isfinite(lse[0, :, 0]).all()
        assert (out[0, :, 1] == 0).all() and (lse[0, :, 1] == -math.inf).all()


def test_shared_pages_are_read_by_both():
    """Two sequences whose tables name the same pages (a prompt in common)."""
    cfg, cache, table, k, v, q = small()
    table[1] = table[0]
    q[1] = q[0]
    o, _ = e2ttt.cache_attention(cfg, dev(q, "bf16"), cache, table, i32([299, 299, 0]))
    assert torch.equal(o[0], o[1])


def test_graph_of_decode_steps_and_other_stream():
    """A step (write, then attention) captured once and replayed while the positions
    move on, against eager calls on another stream and their own cache."""
    cfg, cache, table, _, _, _ = small(P=3, held=60, n=12, left=120)
    mine = cache.clone()
    g = torch.Generator(device="cuda").manual_seed(4)
    dt = torch.bfloat16
    bufs = [torch.empty(3, h, 1, 64, dtype=dt, device="cuda") for h in (4, 2, 2)]
    starts, out = i32([60, 60, 60]), torch.empty(3, 4, 1, 64, dtype=dt, device="cuda")
    ws = e2ttt.alloc_cache_workspace(cfg)

    def step(cache, starts, q, k, v, out, ws):
        e2ttt.cache_write(cfg, k, v, cache, table, starts)
        e2ttt.cache_attention(cfg, q, cache, table, starts, out=out, workspace=ws)

    for b in bufs:
        b.zero_()
    step(cache.clone(), starts, *bufs, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, starts, *bufs, out, ws)
    other = torch.cuda.Stream()
    for i in range(150):
        new = [torch.randn(b.shape, device="cuda", generator=g).to(dt) for b in bufs]
        for b, x in zip(bufs, new):
            b.copy_(x)
        starts.fill_(60 + i)
        at = i32([60 + i] * 3)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(other):
            ref = torch.empty_like(out)
            step(mine, at, *new, ref, e2ttt.alloc_cache_workspace(cfg))
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i
    assert torch.equal(cache, mine)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("P", [2, 70])      # (70 pages are split)
@pytest.mark.parametrize("how", ["up", "down", "raw"])
def test_scores_out_of_range(P, how, io):
    """Finite queries and keys whose scores pass the range of fp32, as q . k or times the
    scale: NaN, and not the zeros of a token that sees no key; those keep theirs."""
    n, T = 64 * P - 3, 2
    cfg = e2ttt.CacheConfig(3, 1, 3, T, 64, P, IO(io), scale=2.0 ** 127 if how != "raw" else 1.0)
    fill = e2ttt.CacheConfig(3, 1, 3, n, 64, P, IO(io))
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    cache, table = e2ttt.alloc_cache(cfg, 3 * P), table_of(3, P, 3 * P).to(torch.int32).cuda()
    k = torch.full((3, 1, n, 64), dict(up=1.0, down=-1.0, raw=-1e25)[how], dtype=dt, device="cuda")
    e2ttt.cache_write(fill, k, torch.randn(k.shape, device="cuda").to(dt), cache, table)
    table[1] = -1
    q = torch.full((3, 3, T, 64), 1e25 if how == "raw" else 1.0, dtype=dt, device="cuda")
    lse = torch.zeros(3, 3, T, device="cuda")
    out, _ = e2ttt.cache_attention(cfg, q, cache, table, i32([n - 2, n - 2, n - 1]), i32([2, 2, 1]), lse=lse)
    assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
    assert torch.isnan(out[2, :, 0]).all() and torch.isnan(lse[2, :, 0]).all()
    for o, l in ((out[1], lse[1]), (out[2, :, 1], lse[2, :, 1])):
        assert (o == 0).all() and (l == -math.inf).all()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("P", [4, 70])
def test_keys_whose_scores_vanish_below_the_range(P, io):
    """Pages, and whole stretches of them, with q . k below fp32's range weigh nothing
    beside the other keys."""
    n, d = 64 * P, 64
    m = n // 2 + 5
    cfg = e2ttt.CacheConfig(1, 1, 2, 1, d, P, IO(io))
    fill = e2ttt.CacheConfig(1, 1, 2, n, d, P, IO(io))
    v = rounded(torch.randn(1, 1, n, d, generator=torch.Generator().manual_seed(7), dtype=torch.float64), io)
    k = torch.zeros_like(v)
    k[:, :, :m, 0] = -2.0 ** 80
    cache, table = e2ttt.alloc_cache(cfg, P), table_of(1, P, P).to(torch.int32).cuda()
    e2ttt.cache_write(fill, dev(k, io), dev(v, io), cache, table)
    q = torch.zeros(1, 2, 1, d, dtype=torch.float64)
    q[..., 0] = 2.0 ** 80
    lse = torch.zeros(1, 2, 1, device="cuda")
    out, _ = e2ttt.cache_attention(cfg, dev(q, io), cache, table, i32([n - 1]), lse=lse)
    held = cacheref.values(*cacheref.quantise(v))[0, 0, m:]
    # (weights of 2^0, sums of n terms, the out's rounding)
    lim = 2.0 ** -24 * (n + 16) * held.abs().mean(0) + (2.0 ** -8 if io == "bf16" else 2.0 ** -23) * held.mean(0).abs()
    assert ((out[0, :, 0].double().cpu() - held.mean(0)).abs() <= 1.01 * lim).all()
    assert (lse.double().cpu() - math.log(n - m)).abs().max() <= 2.0 ** -20


def test_a_window_beyond_half_of_the_positions():
    """left of 2^30 and more: a key that far back is seen, the one before it is not."""
    P, left, start, d = 2 ** 24 + 2, 2 ** 30 + 10, 2 ** 30 + 100, 32
    table = torch.full((1, P), -1, dtype=torch.int32, device="cuda")
    table[0, 1], table[0, start // 64] = 0, 1                # positions 64 .. 127 and the last ones
    g = torch.Generator().manual_seed(3)
    k, v, q = (rounded(torch.randn(1, 1, 64, d, generator=g, dtype=torch.float64), "f32") for _ in "kvq")
    at = lambda T: e2ttt.CacheConfig(1, 1, 1, T, d, P, e2ttt.DT_F32, left=left)
    cache = e2ttt.alloc_cache(at(1), 2)
    e2ttt.cache_write(at(64), dev(k, "f32"), dev(v, "f32"), cache, table, i32([64]))
    n = start % 64 + 1
    e2ttt.cache_write(at(n), dev(k.flip(2)[:, :, :n], "f32"), dev(v.flip(2)[:, :, :n], "f32"), cache, table,
                      i32([start + 1 - n]))
    lse = torch.zeros(1, 1, 1, device="cuda")
    out, _ = e2ttt.cache_attention(at(1), dev(q[:, :, :1], "f32"), cache, table, i32([start]), lse=lse)
    kv = [cacheref.values(*cacheref.quantise(x))[0] for x in (k, v)]
    kv = tuple(torch.cat([x[:, start - left - 64:], x.flip(1)[:, :n]], 1) for x in kv)
    m = kv[0].shape[1]
    ref, ls, bounds = cacheref.attend(q[:, :, :1], [kv], [m - 1], [1], 2, -1, 1.0)
    bo, bl = bounds(False)
    within("out", out, ref, bo, 2.0 ** -18)
    within("lse", lse, ls, bl, 2.0 ** -18)
