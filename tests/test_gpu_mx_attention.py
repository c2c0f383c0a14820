"""Attention over the 4-bit key/value cache on the GPU, against float64.

The bound (mx_cache_reference.tolerance).  A score is a sum of d products that are exact, in chunks whose sums are truncated to
float32 at worst (2^-23 of the magnitudes so far, each), times factors that are powers of two and the scale: off by at most
(2 d + 32) 2^-23 of the largest sum of magnitudes; the exponential adds 2^-22 of the weight and what its argument's rounding makes, in
all 2^-21.  A weight is rounded to float16, 2^-11 of it, or 2^-34 of the largest possible weight if it is small (n of them, of
values up to twice the largest and weights up to 2^0: n 2^-32 vmax with room).  Sums over n tokens: a warp adds n / 64 steps, four
warps and up to some hundred parts are joined: (n / 16 + 64) 2^-23.  A weight's relative error counts twice, in the sum and in what
it is divided by.  Then half a unit of the output: 2^-8 of bfloat16, 2^-23 of float32 with its division."""
import math

import numpy as np
import pytest
import torch

import mx_cache_reference as C

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")
DEV = "cuda"


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


class Batch:
    """Sequences of `lens` tokens with `rows` queries each in a cache of poisoned pages (every scale NaN where no token is)."""

    def __init__(self, seed, lens, rows, hq, hkv, d, page, spare=3, size=1.0, fill=0xFF):
        rng = np.random.default_rng(seed)
        self.rng, self.d, self.page, self.hq, self.hkv = rng, d, page, hq, hkv
        self.lens, self.rows = np.array(lens, dtype=np.int32), np.array(rows)
        count = [-(-max(int(n), 0) // page) for n in lens]
        pages = sum(count) + spare
        order = rng.permutation(pages).astype(np.int32)
        # (few rows times a narrow table are all the first kernel's: ragged batches have room behind their sequences, `narrow` none)
        width = max(count + [1]) + 1
        self.narrow = width
        if sum(rows) > len(rows):
            width += 2 ** 22 // (sum(rows) * hq * page)
        self.table = np.full((len(lens), width), -7, dtype=np.int32)           # (behind a length: not read)
        at = 0
        for s, c in enumerate(count):
            self.table[s, :c] = order[at:at + c]
            at += c
        self.cache = dev(C.blank(pages, hkv, page, d, fill))
        slots = np.concatenate([self.table[s, np.arange(n) // page] * page + np.arange(n) % page for s, n in enumerate(lens) if n > 0]
                               + [np.zeros(0, dtype=np.int64)]).astype(np.int32)
        k = rng.standard_normal((len(slots), hkv, d)) * (1 + 7 * (np.arange(d) < 2)) * size
        v = rng.standard_normal((len(slots), hkv, d)) + 0.25
        if len(slots):
            cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots), self.cache)
        self.offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.q = dev(1.5 * rng.standard_normal((int(sum(rows)), hq, d)), torch.bfloat16)

    def run(self, scale=None, **more):
        scale = self.d ** -0.5 if scale is None else scale
        offsets = more.pop("offsets", self.offsets)
        table = self.table[:, :self.narrow] if more.pop("narrow", False) else self.table
        return cat.cat_mx_attention(self.q, self.cache, dev(np.ascontiguousarray(table)), dev(self.lens), scale,
                                    offsets=None if offsets is None else dev(offsets), **more)

    def check(self, got, scale=None, window=0, offsets="own"):
        scale = self.d ** -0.5 if scale is None else scale
        want = C.attention(host(self.q), host(self.cache), self.page, self.table, self.lens, scale,
                           self.offsets if isinstance(offsets, str) else offsets, window)
        tol = C.tolerance(*want, self.d, got.dtype is torch.bfloat16)
        g = host(got)
        assert g.shape == want[0].shape and np.isfinite(g).all()
        worst = np.max(np.abs(g - want[0]) / tol)
        assert worst <= 1, worst
        return want[0]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv,page", [(1, 1, 16), (4, 1, 64), (8, 8, 32), (10, 2, 16), (16, 1, 128), (24, 8, 1024), (9, 3, 64)])
def test_one_token_each(hq, hkv, page, d):
    b = Batch(hq * d, [1, 2, 15, 16, 17, 0, 31, 33, 64, 65, 200, 999], [1] * 12, hq, hkv, d, page)
    b.check(b.run())
    b.check(b.run(offsets=None, out_dtype=torch.float32))
    b.check(b.run(window=20), window=20)
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (5, 1), (16, 2), (32, 1)])
def test_several_tokens(hq, hkv, d):
    """Rows that see nothing (a sequence shorter than its rows), none at all, more than a tile."""
    b = Batch(hq + d, [5, 40, 300, 3, 0, 17, 130, 16], [5, 3, 7, 6, 2, 0, 40, 1], hq, hkv, d, 32)
    want = b.check(b.run())
    assert not want[15:18].any()                     # tokens -3 .. -1 of a sequence of 3
    for window in (1, 7, 16, 33, 100000):
        b.check(b.run(window=window, out_dtype=torch.float32), window=window)


@pytest.mark.parametrize("d", [64, 256])
def test_a_length_behind_the_table(d):
    """Tokens that no entry of the table is for are not attended, by either kernel."""
    b = Batch(26 + d, [4500, 30, 4120], [200, 3, 2], 8, 2, d, 1024)
    for width in (4, 3, 0):
        b.table = np.ascontiguousarray(b.table[:, :width])
        for window in (0, 300):
            got = host(b.run(window=window, out_dtype=torch.float32))
            if width == 0:
                assert not got.any()
            else:
                want = C.attention(host(b.q), host(b.cache), b.page, b.table, b.lens, d ** -0.5, b.offsets, window)
                assert np.all(np.abs(got - want[0]) <= C.tolerance(*want, d, False))
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv,lens,rows", [
    (8, 2, [5, 40, 300, 3, 0, 17, 130, 16], [5, 3, 7, 6, 2, 0, 40, 1]), (20, 4, [7, 7, 5], [7, 6, 5]), (4, 4, [500], [300]),
    (64, 1, [33, 100], [1, 2]), (5, 1, [1], [1]), (9, 3, [700, 20], [30, 20])])
def test_many_rows_with_a_narrow_table(hq, hkv, lens, rows, d):
    """(All of them the first kernel's, some of several tiles; beside them, with room in the table, the second's.)"""
    b = Batch(25 + hq + d, lens, rows, hq, hkv, d, 16)
    for window in (0, 1, 9, 64):
        b.check(b.run(window=window, narrow=True), window=window)
        b.check(b.run(window=window, out_dtype=torch.float32), window=window)
    got = b.run(narrow=True)
    assert torch.equal(got, b.run(narrow=True))
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("hq,hkv,d,lens,rows", [
    (32, 8, 128, [70001], [1]), (2, 1, 64, [40000, 3, 12345], [1, 1, 1]), (4, 2, 256, [9000, 20000], [1, 2]),
    (16, 8, 128, [4097] * 9, [1] * 9), (8, 1, 128, [5000, 0, 7000], [4, 4, 5]), (64, 8, 128, list(range(1, 400, 7)), [1] * 57),
    (6, 6, 64, [0] * 40 + [513] * 30, [1] * 70)])
def test_work_cut_over_the_device(hq, hkv, d, lens, rows):
    b = Batch(len(lens) + d, lens, rows, hq, hkv, d, 64)
    got = b.run()
    b.check(got)
    assert torch.equal(got, b.run())                 # the same bits each time


@pytest.mark.parametrize("hq,hkv,d,q,length,window", [(4, 2, 128, 130, 130, 0), (8, 2, 64, 200, 333, 0), (3, 1, 256, 70, 200, 50),
                                                      (2, 2, 128, 300, 301, 64), (5, 1, 64, 129, 129, 1)])
def test_prompts(hq, hkv, d, q, length, window):
    b = Batch(q, [length, 40, 7], [q, 33, 1], hq, hkv, d, 16)
    b.check(b.run(window=window), window=window)
    b = Batch(q, [length], [q], hq, hkv, d, 64)
    b.check(b.run(window=window), window=window)
    b.check(b.run(window=window, out_dtype=torch.float32), window=window)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv,page,lens,rows,window", [
    (4, 1, 64, [1000, 0, 333, 64, 2000], [500, 3, 333, 40, 1], 0), (40, 1, 16, [200, 90, 17], [1, 1, 1], 0), (3, 3, 128, [700, 650], [700, 128], 100),
    (16, 2, 1024, [3000], [70], 0), (5, 1, 32, [400, 30], [257, 60], 0), (17, 1, 16, [5, 300], [9, 2], 33), (8, 2, 64, [129, 127, 128], [129, 127, 64], 0)])
def test_tiles(hq, hkv, page, lens, rows, window, d):
    """Sequences of many rows beside others: whole tiles and parts of them, rows that see nothing, groups that no tile's rows divide."""
    b = Batch(d + hq, lens, rows, hq, hkv, d, page)
    got = b.run(window=window)
    b.check(got, window=window)
    assert torch.equal(got, b.run(window=window))
    b.check(b.run(window=window, out_dtype=torch.float32), window=window)
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("scale", [0.0, -0.3, 20.0])
def test_tiles_scales_and_sizes(scale):
    b = Batch(19, [500, 90], [200, 90], 4, 2, 128, 32)
    b.check(b.run(scale=scale), scale=scale)
    n = 500
    for up in (1, -1):
        v = b.rng.standard_normal((n, 2, 128)) * np.exp2(up * np.linspace(-20, 20, n))[:, None, None]
        v[:, :, 32:64] *= 2.0 ** -12
        k = b.rng.standard_normal((n, 2, 128)) * np.exp2(2 * np.sin(np.arange(n)))[:, None, None]
        slots = b.table[0, np.arange(n) // 32] * 32 + np.arange(n) % 32
        cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots.astype(np.int32)), b.cache)
        b.check(b.run(scale=scale / 4), scale=scale / 4)


def test_tiles_of_a_long_sequence():
    """Units cut into parts, and pages that are none."""
    b = Batch(21, [20000, 300], [70, 2], 8, 1, 128, 64)
    b.table[0, 7], b.table[0, 150] = -1, 10 ** 6
    got = b.run()
    b.check(got)
    assert torch.equal(got, b.run())


def test_many_sequences():
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 40, 700)
    b = Batch(11, lens.tolist(), [1] * 700, 4, 2, 64, 16)
    b.check(b.run(offsets=None))


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 40.0])
def test_scales(scale):
    b = Batch(5, [100, 1000], [2, 3], 4, 2, 128, 32)
    b.check(b.run(scale=scale), scale=scale)


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 40])
def test_queries_far_from_one(size):
    b = Batch(6, [100, 500], [1, 3], 4, 2, 128, 32)
    b.q = b.q * size
    b.q[1] = 0.0
    b.check(b.run(scale=0.1 / size), scale=0.1 / size)


def test_values_of_many_sizes():
    """Blocks whose scales are far apart, in either order along a sequence."""
    for up in (1, -1):
        b = Batch(7, [600, 90], [1, 2], 4, 2, 128, 16)
        n = 600
        v = b.rng.standard_normal((n, 2, 128)) * np.exp2(up * np.linspace(-20, 20, n))[:, None, None]
        v[:, :, 32:64] *= 2.0 ** -30
        k = b.rng.standard_normal((n, 2, 128))
        slots = b.table[0, np.arange(n) // 16] * 16 + np.arange(n) % 16
        cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots.astype(np.int32)), b.cache)
        b.check(b.run())


def test_rows_before_and_behind_the_sequences_are_zero():
    b = Batch(8, [20, 50], [3, 4], 4, 2, 64, 16)
    b.q = torch.cat([b.q, b.q, b.q])
    offsets = np.array([2, 5, 9], dtype=np.int32)
    out = torch.full((21, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    assert b.run(offsets=offsets, out=out) is out
    want = b.check(out, offsets=offsets)
    assert not want[:2].any() and not want[9:].any()
    # offsets outside the rows are taken as the nearest that are not
    b.check(b.run(offsets=np.array([-5, 4, 90], dtype=np.int32)), offsets=np.array([0, 4, 21]))


def test_no_sequences():
    q = torch.ones((3, 4, 64), dtype=torch.bfloat16, device=DEV)
    cache = cat.cat_mx_cache(1, 2, 16, 64)
    none = torch.zeros((0, 5), dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 5.0)
    cat.cat_mx_attention(q, cache, none, none[:, 0].contiguous(), 1.0, offsets=torch.zeros(1, dtype=torch.int32, device=DEV), out=out)
    assert not out.any()
    empty = cat.cat_mx_attention(q[:0], cache, none, none[:, 0].contiguous(), 1.0)
    assert empty.shape == (0, 4, 64)


def test_pages_that_are_none_hold_no_tokens():
    b = Batch(9, [200, 64, 30], [2, 1, 1], 4, 2, 128, 16)
    b.table[0, 3], b.table[0, 5], b.table[0, 12] = -1, 10 ** 6, b.cache.shape[0]
    b.table[1, :] = -1
    want = b.check(b.run())
    assert not want[2].any()
    # tokens past a table's end
    b = Batch(10, [100], [1], 4, 2, 64, 16)
    b.table = b.table[:, :3]
    b.check(b.run())
    b.check(b.run(window=60), window=60)


def test_nan_of_tokens_that_are_not_seen():
    """NaN keys and values ahead of a row, behind its window, and of a token that some rows of a tile see and others do not."""
    b = Batch(12, [90, 40], [6, 4], 4, 2, 128, 32)
    bad = np.full((2, 2, 128), np.nan)
    t = np.array([20, 88])                                         # behind the windows; seen by the last two rows of six
    slots = (b.table[0, t // 32] * 32 + t % 32).astype(np.int32)
    cat.cat_mx_cache_write(dev(bad, torch.float32), dev(bad, torch.float32), dev(slots), b.cache)
    cat.cat_device_status()
    got = b.run(window=30)
    want = C.attention(host(b.q), host(b.cache), b.page, b.table, b.lens, b.d ** -0.5, b.offsets, 30)
    tol = C.tolerance(*want, b.d, True)
    g = host(got)
    fine = [0, 1, 2, 3, 6, 7, 8, 9]
    assert np.all(np.abs(g - want[0])[fine] <= tol[fine])
    assert np.isnan(g[4:6]).all()
    # values alone
    b = Batch(13, [90], [6], 4, 2, 128, 32)
    slots = (b.table[0, t // 32] * 32 + t % 32).astype(np.int32)
    k = b.rng.standard_normal((2, 2, 128))
    v = np.ones((2, 2, 128))
    v[:, 1, 40] = np.inf
    cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots), b.cache)
    cat.cat_device_status()
    g = host(b.run(window=30))
    assert np.isfinite(g[:4]).all() and np.isnan(g[4:, 2:, 32:64]).all()
    assert np.isfinite(g[4:, :2]).all() and np.isfinite(g[4:, 2:, :32]).all() and np.isfinite(g[4:, 2:, 64:]).all()


@pytest.mark.parametrize("rows", [[1, 1, 3], [40, 20, 33]])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_is_not_seen_may_be_anything(d, rows):
    """Cache rows behind the lengths of the largest finite scales and codes; tokens behind the window of the largest values."""
    b = Batch(17, [90, 40, 150], rows, 8, 2, d, 64, fill=0xFD)
    b.check(b.run())
    k = np.full((30, 2, d), 2.0 ** 120)
    slots = (b.table[2, np.arange(30) // 64] * 64 + np.arange(30) % 64).astype(np.int32)
    cat.cat_mx_cache_write(dev(k, torch.float32), dev(k, torch.float32), dev(slots), b.cache)
    b.check(b.run(window=80), window=80)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_nan_of_tokens_that_a_prompts_rows_do_not_see(d):
    b = Batch(18, [300, 70], [200, 70], 4, 2, d, 32)
    t = np.array([20, 230])                                        # behind the windows of all; seen from row 130 on, to row 159
    slots = (b.table[0, t // 32] * 32 + t % 32).astype(np.int32)
    k, v = b.rng.standard_normal((2, 2, d)), np.ones((2, 2, d))
    v[:, 1, 40] = np.inf
    cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots), b.cache)
    cat.cat_device_status()
    want = C.attention(host(b.q), host(b.cache), b.page, b.table, b.lens, d ** -0.5, b.offsets, 30)
    tol = C.tolerance(*want, d, True)
    g = host(b.run(window=30))
    odd = np.zeros(g.shape, dtype=bool)
    odd[130:160, 2:, 32:64] = True
    assert np.isnan(g[odd]).all() and np.isfinite(g[~odd]).all()
    assert np.all(np.abs(g - want[0])[~odd] <= tol[~odd])
    bad = np.full((2, 2, d), np.nan)                               # keys too
    cat.cat_mx_cache_write(dev(bad, torch.float32), dev(v, torch.float32), dev(slots), b.cache)
    cat.cat_device_status()
    g = host(b.run(window=30))
    odd[:] = False
    odd[130:160] = True
    assert np.isnan(g[odd]).all() and np.isfinite(g[~odd]).all()
    assert np.all(np.abs(g - want[0])[~odd] <= tol[~odd])


def test_queries_that_are_not_finite():
    b = Batch(14, [50, 60], [3, 1], 4, 2, 64, 16)
    b.q[1, 2, 5], b.q[3, 0, 0] = float("nan"), float("inf")
    g = host(b.run())
    odd = np.zeros((4, 4), dtype=bool)
    odd[1, 2] = odd[3, 0] = True
    assert np.isnan(g[odd]).all() and np.isfinite(g[~odd]).all()
    b.q[1, 2, 5], b.q[3, 0, 0] = 0.0, 0.0
    g[odd] = 0.0
    again = host(b.run())
    assert np.array_equal(g[~odd], again[~odd])


def test_streams_and_graphs():
    """Calls on two streams at once; a captured call replayed with other lengths, beside calls of its kind."""
    a, b = Batch(15, [3000, 5000], [1, 1], 8, 2, 128, 64), Batch(16, [4000], [2], 16, 4, 64, 16)
    wa, wb = a.run(), b.run()
    table, lens, offsets = dev(a.table), dev(a.lens), dev(a.offsets)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(10):
        with torch.cuda.stream(s1):
            outs.append((cat.cat_mx_attention(a.q, a.cache, table, lens, 128 ** -0.5, offsets=offsets), wa))
        with torch.cuda.stream(s2):
            outs.append((b.run(), wb))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in outs)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = cat.cat_mx_attention(a.q, a.cache, table, lens, 128 ** -0.5, offsets=offsets)
        graphs.append((g, o))
    lens.copy_(torch.tensor([17, 2500], dtype=torch.int32))
    torch.cuda.synchronize()
    for s, (g, _) in zip((s1, s2), graphs):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    a.lens = np.array([17, 2500], dtype=np.int32)
    a.check(graphs[0][1])
    assert torch.equal(graphs[0][1], graphs[1][1])


def test_prompts_on_streams_and_in_graphs():
    """Both kernels of a mixed batch, on two streams at once and replayed with other lengths."""
    a = Batch(22, [400, 700, 90], [200, 1, 2], 8, 2, 128, 64)
    b = Batch(23, [900], [300], 4, 1, 64, 16)
    wa, wb = a.run(), b.run()
    a.check(wa)
    table, lens, offsets = dev(a.table), dev(a.lens), dev(a.offsets)
    bt, bl, bo = dev(b.table), dev(b.lens), dev(b.offsets)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(8):
        with torch.cuda.stream(s1):
            outs.append((cat.cat_mx_attention(a.q, a.cache, table, lens, 128 ** -0.5, offsets=offsets), wa))
        with torch.cuda.stream(s2):
            outs.append((cat.cat_mx_attention(b.q, b.cache, bt, bl, 64 ** -0.5, offsets=bo), wb))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in outs)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        oa = cat.cat_mx_attention(a.q, a.cache, table, lens, 128 ** -0.5, offsets=offsets)
        ob = cat.cat_mx_attention(b.q, b.cache, bt, bl, 64 ** -0.5, offsets=bo)
    lens.copy_(torch.tensor([250, 64, 90], dtype=torch.int32))
    offsets.copy_(torch.tensor([0, 130, 131, 203], dtype=torch.int32))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    a.lens, a.offsets = np.array([250, 64, 90], dtype=np.int32), np.array([0, 130, 131, 203], dtype=np.int32)
    a.check(oa)
    assert torch.equal(ob, wb)
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("offsets", [[5, 2, 9, 300], [0, 400, -3, 7], [250, 240, 10, 0]])
def test_offsets_out_of_order_stay_within_the_rows(offsets):
    """(Which sequence a row named twice is of is not said; nothing outside is written, and the next call is right.)"""
    b = Batch(24, [300, 50, 400], [100, 60, 100], 4, 2, 128, 32)
    room = torch.full((262, 4, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    b.run(offsets=np.array(offsets, dtype=np.int32), out=room[1:261])
    assert bool((room[0] == 3).all()) and bool((room[261] == 3).all())
    b.check(b.run())


def test_a_decode_loop():
    """Prompts and steps as a server runs them: projections' rows through norms and rotation into the cache, attention behind."""
    rng = np.random.default_rng(20)
    hq, hkv, d, page, steps = 8, 2, 128, 16, 5
    prompt = [30, 7, 16]
    cos, sin = (dev(f(np.arange(64)[:, None] * 100.0 ** (-np.arange(d // 2) / (d // 2))), torch.float32) for f in (np.cos, np.sin))
    wq, wk = dev(1 + 0.1 * rng.standard_normal(d), torch.bfloat16), dev(1 + 0.1 * rng.standard_normal(d), torch.bfloat16)
    width = 4
    table = rng.permutation(3 * width).reshape(3, width).astype(np.int32)
    cache = cat.cat_mx_cache(3 * width, hkv, page, d)
    past = [[], [], []]
    lens = np.zeros(3, dtype=np.int32)
    for step in range(steps + 1):
        rows = prompt if step == 0 else [1, 1, 1]
        pos = np.concatenate([np.arange(lens[s], lens[s] + rows[s]) for s in range(3)]).astype(np.int32)
        owner = np.repeat(np.arange(3), rows)
        slots = (table[owner, pos // page] * page + pos % page).astype(np.int32)
        qkv = dev(rng.standard_normal((len(pos), (hq + 2 * hkv) * d)), torch.bfloat16)
        q = cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, q_weight=wq, k_weight=wk)
        lens = (lens + np.array(rows)).astype(np.int32)
        offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        got = cat.cat_mx_attention(q, cache, dev(table), dev(lens), d ** -0.5, offsets=dev(offsets) if step == 0 else None)
        want = C.attention(host(q), host(cache), page, table, lens, d ** -0.5, offsets)
        assert np.all(np.abs(host(got) - want[0]) <= C.tolerance(*want, d, True))
        # and the cache is what the rows' float64 keys and values give
        x = host(qkv).reshape(len(pos), -1, d)
        k = C.turned(C.normed(x[:, hq:hq + hkv], host(wk), 1e-6), host(cos)[pos], host(sin)[pos], False)
        for i, s in enumerate(owner):
            past[s].append((k[i], x[i, hq + hkv:]))
    for s in range(3):
        k, v = (np.stack([p[i] for p in past[s]]) for i in (0, 1))
        t = np.arange(len(past[s]))
        slots = table[s, t // page] * page + t % page
        want = C.store(C.blank(3 * width, hkv, page, d), page, k, v, slots)
        for kind in (0, 1):
            np.testing.assert_array_equal(C.load(host(cache), page, d, slots, kind), C.load(want, page, d, slots, kind))
