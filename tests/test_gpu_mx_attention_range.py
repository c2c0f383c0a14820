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


def grown(b, s, at, size, kind):
    """The token's keys or values a size larger."""
    t = np.array([at])
    x = b.rng.standard_normal((1, b.cache.shape[2], b.d)) * size
    rewrite(b, s, t, **{kind: x})
