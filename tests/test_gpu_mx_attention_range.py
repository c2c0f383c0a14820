"""Attention over the 4-bit key/value cache at the ends of float32's range, and what a row's result may depend on.

The bound is test_gpu_mx_attention.py's, but for its part of small weights: of the largest value that the row itself sees."""
import numpy as np
import pytest
import torch

import mx_cache_reference as C
from test_gpu_mx_attention import Batch, dev, host

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")

FEW, TILES, BOTH = [1, 3, 2], [200, 40, 70], [200, 1, 3]


def rewrite(b, s, t, k=None, v=None):
    """Tokens t of sequence s get keys k and values v [len(t), hkv, d]; None keeps what is there."""
    slots = (b.table[s, t // b.page] * b.page + t % b.page).astype(np.int32)
    old = C.load(host(b.cache), b.page, b.d, slots, 0), C.load(host(b.cache), b.page, b.d, slots, 1)
    k, v = (o if x is None else x for o, x in zip(old, (k, v)))
    cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots), b.cache)


def seen_vmax(b, window):
    """The largest magnitude of a value that each row sees."""
    out = np.zeros(b.q.shape[0])
    at = 0
    for s, rows in enumerate(b.rows):
        t = np.arange(b.lens[s])
        most = np.abs(C.load(host(b.cache), b.page, b.d, b.table[s, t // b.page] * b.page + t % b.page, 1)).max(axis=(1, 2)) if len(t) else t
        for j in range(rows):
            p = b.lens[s] - rows + j
            seen = (t <= p) & ((t > p - window) if window else True)
            out[at] = most[seen].max() if seen.any() else 0.0
            at += 1
    return out


def check(b, scale=None, window=0, **more):
    scale = b.d ** -0.5 if scale is None else scale
    got = host(b.run(scale=scale, window=window, out_dtype=torch.float32, **more))
    out, mass, dots, _, count = C.attention(host(b.q), host(b.cache), b.page, b.table, b.lens, scale, b.offsets, window)
    # (a row whose weights the bound says nothing of is checked for being finite alone)
    with np.errstate(over="ignore", invalid="ignore"):
        tol = C.tolerance(out, mass, dots, seen_vmax(b, window), count, b.d, False)
    assert np.isfinite(got).all(), f"rows {np.unique(np.nonzero(~np.isfinite(got))[0])[:10]}"
    off = np.abs(got - out) / tol
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert off[worst] <= 1, (off[worst], worst, got[worst], out[worst])


@pytest.mark.parametrize("rows", [FEW, TILES])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** -118, 2.0 ** -70, 2.0 ** 70, 2.0 ** 108, 2.0 ** 121])
def test_keys_far_from_one(size, d, rows):
    b = Batch(31 + d, [300, 90, 150], rows, 8, 2, d, 32, size=size)
    check(b, scale=d ** -0.5 / size)


@pytest.mark.parametrize("rows", [FEW, TILES])
@pytest.mark.parametrize("size,key", [(2.0 ** -120, 2.0 ** 4), (2.0 ** 120, 2.0 ** -4), (2.0 ** -60, 2.0 ** -58), (2.0 ** 100, 2.0 ** -100),
                                      (2.0 ** -100, 2.0 ** 110)])
def test_queries_and_keys_far_from_one(size, key, rows):
    b = Batch(32, [300, 90, 150], rows, 4, 2, 128, 32, size=key)
    b.q = b.q * size
    b.q[0] = 0.0
    b.q[3:5] = b.q[3:5] / size
    scale = np.sqrt(1 / 128) / size / key
    with np.errstate(over="ignore"):
        ok = abs(np.float32(scale * 2)) < np.finfo(np.float32).max
    check(b, scale=scale if ok else 2.0 ** 127)


@pytest.mark.parametrize("lens,rows,hq", [([1, 200, 90], [1, 2, 1], 8), ([300, 90], [200, 40], 8), ([9000], [1], 8), ([9000, 20], [3, 1], 8),
                                          ([20000], [70], 8), ([5000, 4000], [150, 1], 4)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** -108, 2.0 ** -80, 2.0 ** 112, 2.0 ** 124])
def test_values_far_from_one(size, d, lens, rows, hq):
    """(Long sequences' units are cut in parts.)"""
    if d == 256 and lens[0] > 9000:
        lens = [9000]
    b = Batch(33 + d, lens, rows, hq, 1, d, 64)
    b.q = b.q * 0.25                                               # (many weights of a size)
    for s, n in enumerate(lens):
        rewrite(b, s, np.arange(n), v=(b.rng.uniform(-1.0, 1.0, (n, 1, d)) + 0.5) * size)
    check(b)


def grown(b, s, at, size, kind):
    """The token's keys or values a size larger."""
    t = np.array([at])
    x = b.rng.standard_normal((1, b.cache.shape[2], b.d)) * size
    rewrite(b, s, t, **{kind: x})


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** 14, 2.0 ** 26, 2.0 ** 60, 2.0 ** 110])
@pytest.mark.parametrize("rows,window", [([6, 3, 2], 0), ([6, 3, 2], 40), ([6, 3, 2], 2), ([6, 3, 6], 32), ([200, 40, 70], 0),
                                         ([200, 40, 70], 40), ([200, 1, 8], 33), ([200, 30, 70], 2)])
def test_values_that_some_rows_see(rows, window, size, d):
    """A value of another size ahead of a batch's early rows, and one behind its late rows' windows."""
    b = Batch(34 + d, [300, 90, 150], rows, 4, 2, d, 32)
    for s, (n, r) in enumerate(zip(b.lens, rows)):
        grown(b, s, n - r + r // 2, size, "v")
        if window:
            grown(b, s, max(n - window - r // 2, 0), size, "v")
    check(b, window=window)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [2.0 ** 26, 2.0 ** 60])
@pytest.mark.parametrize("rows,window", [([6, 3, 2], 0), ([200, 40, 70], 0), ([200, 40, 70], 40)])
def test_keys_that_some_rows_see(rows, window, size, d):
    b = Batch(35 + d, [300, 90, 150], rows, 8, 2, d, 32)
    for s, (n, r) in enumerate(zip(b.lens, rows)):
        grown(b, s, n - r + r // 2, size, "k")
        if window:
            grown(b, s, max(n - window - r // 2, 0), size, "k")
    check(b, window=window)


@pytest.mark.parametrize("rows,lens", [([1, 1, 1], [1, 40, 5000]), ([200, 40], [300, 3000])])
@pytest.mark.parametrize("size", [-1.0, 1.0])
def test_scores_of_any_size(size, rows, lens):
    """Equal scores are equal weights, whatever they are: here 2^112 and -2^112."""
    d = 128
    b = Batch(36, lens, rows, 8, 2, d, 32)
    b.q = torch.ones_like(b.q)
    for s, n in enumerate(lens):
        rewrite(b, s, np.arange(n), k=np.full((n, 2, d), 2.0 ** 50))
    got = host(b.run(scale=size * 2.0 ** 55, out_dtype=torch.float32))
    at = 0
    for s, (n, r) in enumerate(zip(lens, rows)):
        t = np.arange(n)
        v = C.load(host(b.cache), b.page, d, b.table[s, t // b.page] * b.page + t % b.page, 1)
        for j in range(r):
            p = n - r + j + 1
            # (weights of 1 exactly; a sum of p values in float32)
            bound = (p / 16 + 64) * 2.0 ** -23 * np.abs(v[:p]).mean(0)
            assert np.all(np.abs(got[at] - np.repeat(v[:p].mean(0), 4, 0)) <= np.repeat(bound, 4, 0)), (s, j)
            at += 1


@pytest.mark.parametrize("rows", [[1, 3], [200, 40]])
def test_a_nan_value_of_the_smallest_weight(rows):
    """A token that a row sees counts, though its weight is below float32."""
    d = 64
    b = Batch(37, [300, 90], rows, 4, 2, d, 32)
    b.q = torch.ones_like(b.q)
    for s in range(2):
        n = int(b.lens[s])
        k = np.ones((n, 2, d))
        k[7] = -6.0
        v = C.load(host(b.cache), b.page, d, b.table[s, np.arange(n) // b.page] * b.page + np.arange(n) % b.page, 1)
        v[7, 1, 40] = np.nan
        rewrite(b, s, np.arange(n), k=k, v=v)
    cat.cat_device_status()
    g = host(b.run(scale=1.0))
    odd = np.zeros(g.shape, dtype=bool)
    odd[:, 2:, 32:64] = True
    assert np.isnan(g[odd]).all() and np.isfinite(g[~odd]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_tiles_queries_far_from_one_and_not_finite(d):
    """The tiles' way of a query to float16: zero rows, the largest and smallest, NaN and infinity, and the rows beside them."""
    b = Batch(38 + d, [300, 70], [200, 40], 4, 2, d, 32)
    up = torch.ones((240, 4, 1), dtype=torch.float32, device=b.q.device)
    up[3], up[70, 1], up[150, 2], up[239, 3] = 0.0, 2.0 ** 120, 2.0 ** -110, 2.0 ** 123
    b.q = (b.q.float() * up).to(torch.bfloat16)
    for scale in (d ** -0.5, -0.2, 0.0):
        check(b, scale=scale)
    small = 2.0 ** 100
    b.q = (b.q.float() * torch.where(up > 1, 1 / small, 1.0)).to(torch.bfloat16)
    check(b, scale=2.0 ** -20)
    b.q[20, 1, 5], b.q[129, 3, 0] = float("nan"), float("inf")
    g = host(b.run())
    odd = np.zeros((240, 4), dtype=bool)
    odd[20, 1] = odd[129, 3] = True
    assert np.isnan(g[odd]).all() and np.isfinite(g[~odd]).all()
    b.q[20, 1, 5], b.q[129, 3, 0] = 0.0, 0.0
    again = host(b.run())
    assert np.array_equal(g[~odd], again[~odd])


def test_many_sequences_some_of_many_rows():
    """More sequences than the tiles' block has threads, prompts among them."""
    rng = np.random.default_rng(2)
    lens, rows = rng.integers(0, 40, 1300), np.ones(1300, dtype=int)
    rows[::7] = 0
    for s in (0, 575, 576, 577, 900, 1299):
        lens[s], rows[s] = 60 + s % 7, 30 + s % 5
    b = Batch(39, lens.tolist(), rows.tolist(), 4, 2, 64, 16)
    check(b)
    check(b, window=17)


def random_batch(seed):
    """A batch of any kind: prompts, drafted tokens, decode steps; keys and values of sizes that go along, jump or lie far from one."""
    rng = np.random.default_rng(seed)
    d, hkv, group = int(rng.choice([64, 128, 256])), int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 4, 5, 8, 17]))
    page, seqs, kind = int(rng.choice([16, 32, 64, 128])), int(rng.integers(1, 6)), rng.choice(["decode", "draft", "prompt", "mixed"])
    lens = [int(np.exp(rng.uniform(0, np.log(700)))) for _ in range(seqs)]
    if rng.random() < 0.2:
        lens[0] = 3000
    rows = []
    for n in lens:
        k = kind if kind != "mixed" else rng.choice(["decode", "draft", "prompt"])
        rows.append(1 if k == "decode" else int(rng.integers(1, 12)) if k == "draft" else int(rng.integers(1, min(n, 300) + 1)))
    if rng.random() < 0.3:
        rows[0] = min(lens[0] + int(rng.integers(0, 4)), 300)
    b = Batch(seed, lens, rows, hkv * group, hkv, d, page, fill=int(rng.choice([0xFF, 0xFD, 0x00])))
    sizes = {"plain": lambda n, up: np.ones(n), "spread": lambda n, up: np.exp2(rng.uniform(-30, up, n)),
             "jumps": lambda n, up: np.where(rng.random(n) < 0.02, 2.0 ** rng.uniform(0, 2 * up + 1), 1.0),
             "walk": lambda n, up: np.exp2(np.cumsum(rng.normal(0, 1.0, n)).clip(-60, up)),
             "tiny": lambda n, up: np.exp2(rng.uniform(-100, -90, n)),
             "huge": lambda n, up: np.exp2(rng.uniform(90, 118, n)) if up > 5 else np.ones(n)}
    for s, n in enumerate(lens):
        k, v = (rng.standard_normal((n, hkv, d)) * sizes[rng.choice(list(sizes))](n, up)[:, None, None] for up in (2, 60))
        if rng.random() < 0.3:
            v[:, :, 32:64] *= 2.0 ** -20
        if rng.random() < 0.2:
            v[rng.integers(0, n)] = 0.0
            k[rng.integers(0, n)] = 0.0
        rewrite(b, s, np.arange(n), k=k, v=v)
    window = int(np.exp(rng.uniform(0, np.log(800)))) if rng.random() < 0.5 else 0
    return b, dict(window=window, narrow=bool(rng.random() < 0.3), scale=float(d ** -0.5 * rng.choice([1, 1, -1, 4, 0.01])))


@pytest.mark.parametrize("seed", range(48))
def test_random_batches(seed):
    b, how = random_batch(1000 + seed)
    check(b, **how)


@pytest.mark.parametrize("rows", [[2, 40], [100, 40]])
def test_a_rows_values_below_ones_that_it_does_not_see(rows):
    """The largest that a row sees has a weight of 2^-20, and its result is of values as much below that; the next token's are up to 2^10 above."""
    n = rows[0] + 2
    for up in range(1, 11):
        b = Batch(61, [n, 300], rows, 4, 2, 128, 32)
        b.q = torch.ones_like(b.q)
        size, k = np.full((n, 1, 1), 2.0 ** -20), 0.5 * b.rng.standard_normal((n, 2, 128))
        size[0], k[0] = 1.0, -1.0
        size[n - 1], k[n - 1] = 2.0 ** up, -1.0
        rewrite(b, 0, np.arange(n), k=k, v=b.rng.uniform(0.5, 1.0, (n, 2, 128)) * size)
        check(b, scale=14 / 128)
