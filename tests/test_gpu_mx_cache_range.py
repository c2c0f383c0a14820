"""Keys behind norm and rotation at the ends of float32's range: codes are those of the exact value there too."""
import numpy as np
import pytest
import torch

import mx_cache_reference as C
from test_gpu_mx_cache import dev, host, same_cache

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")


def both(qkv, hq, hkv, d, rng, wk=None, rot=None, interleaved=False, turned=True):
    n, page = qkv.shape[0], 64
    rot = rot or d
    pages = -(-n // page)
    angle = rng.uniform(0, 6.3, (100, rot // 2)) * turned
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    pos, slots = rng.integers(0, 100, n).astype(np.int32), rng.permutation(pages * page)[:n].astype(np.int32)
    cache = dev(C.blank(pages, hkv, page, d, 0x11))
    before = host(cache)
    cat.cat_mx_rope_cache_write(dev(qkv), d, dev(pos), dev(cos), dev(sin), dev(slots), cache, k_weight=None if wk is None else dev(wk),
                                interleaved=interleaved)
    x = qkv.astype(np.float64).reshape(n, -1, d)
    k = C.turned(C.normed(x[:, hq:hq + hkv], None if wk is None else wk.astype(np.float64), 1e-6), cos.astype(np.float64)[pos],
                 sin.astype(np.float64)[pos], interleaved)
    same_cache(host(cache), C.store(before, page, k, x[:, hq + hkv:], slots), page, d)


@pytest.mark.parametrize("interleaved", [False, True])
def test_keys_near_a_border_beside_keys_of_another_size(interleaved):
    """A key that is computed again for its borders has beside it, in the same warp, one whose weight times channel leaves float32."""
    rng = np.random.default_rng(41)
    n, hq, hkv, d = 20000, 1, 2, 64
    x = rng.standard_normal((n, hq + 2 * hkv, d)).astype(np.float32)
    wk = np.ones(d, dtype=np.float32)
    wk[40] = 2.0 ** 100
    x[:, 1, 40] = 0.0
    x[:, 1, 41 if interleaved else 8] *= 0.5
    x[:, 2] *= 2.0 ** 40
    both(x.reshape(n, -1), hq, hkv, d, rng, wk, rot=32, interleaved=interleaved)


@pytest.mark.parametrize("size", [2.0 ** -129, 2.0 ** -128, 2.0 ** -126, 2.0 ** -110])
@pytest.mark.parametrize("interleaved,rot", [(False, 64), (True, 64), (False, 16)])
def test_keys_below_float32s_normal_numbers(interleaved, rot, size):
    rng = np.random.default_rng(42)
    n, hq, hkv, d = 20000, 1, 2, 64
    x = (rng.standard_normal((n, hq + 2 * hkv, d)) * size).astype(np.float32)
    both(x.reshape(n, -1), hq, hkv, d, rng, rot=rot, interleaved=interleaved)
