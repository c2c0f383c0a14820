"""The 4-bit key/value cache on the GPU: rows written, read, and written behind head norms and the rotation.

Writing and reading given values is exact: bytes equal the reference's (a value that rounds to zero may keep its sign).  Behind
norm and rotation a key's codes are those of the exact value: the reference's in float64, which is off by some 2^-50, so a code
could differ where the exact value lies that near to a middle -- of the 10^6 values here, none does.  Queries: float32's error is
at most 20 units of 2^-24 of |r w x cos| + |r w' x' sin| (a row's squares 10, the root 2, products and sum 5, and a margin of 3),
then half a unit of bfloat16, 2^-8."""
import numpy as np
import pytest
import torch

import mx_cache_reference as C
import mx_reference as R

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def same_cache(got, want, page, d):
    """Bytes, but for the sign of codes that are zero."""
    gc, gs = C.parts(got, page, d)
    wc, ws = C.parts(want, page, d)
    np.testing.assert_array_equal(gs, ws)

    def unsigned_zero(c):
        lo, hi = c & 15, c >> 4
        return np.where(lo == 8, 0, lo) | (np.where(hi == 8, 0, hi) << 4)
    np.testing.assert_array_equal(unsigned_zero(gc), unsigned_zero(wc))


def heads(rng, n, h, d):
    x = rng.standard_normal((n, h, d)) * np.exp(rng.standard_normal((n, h, 1)))
    x[..., : d // 32] *= 30.0
    if n > 2:
        x[1] = 0.0
        x[2, :, :32] = 0.0
    return x


def some_slots(rng, n, rows):
    s = rng.permutation(rows)[:n].astype(np.int32)
    if n > 4:
        s[3], s[4] = -1, rows                       # a padded batch's, and one behind the cache
    return s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,hkv,d,page", [(1, 1, 64, 16), (1, 8, 128, 64), (5, 3, 128, 32), (7, 1, 256, 16), (27, 12, 64, 1024),
                                          (130, 8, 128, 16), (257, 5, 256, 128), (1000, 2, 64, 64), (3000, 16, 128, 64)])
def test_write_and_read(n, hkv, d, page, dtype):
    rng = np.random.default_rng(n + hkv + d)
    pages = -(-n // page) + 3
    k, v = dev(heads(rng, n, hkv, d), TYPES[dtype]), dev(heads(rng, n, hkv, d) + 0.1, TYPES[dtype])
    slots = some_slots(rng, n, pages * page)
    cache = dev(C.blank(pages, hkv, page, d, 0xA5))
    before = host(cache)
    assert cat.cat_mx_cache_write(k, v, dev(slots), cache) is cache
    want = C.store(before, page, host(k), host(v), slots)
    same_cache(host(cache), want, page, d)
    again = rng.integers(-3, pages * page + 3, size=n + 9).astype(np.int32)          # any order, twice, outside
    for out in TYPES.values():
        gk, gv = cat.cat_mx_cache_read(cache, dev(again), d, out_dtype=out)
        assert gk.dtype is out and gk.shape == (n + 9, hkv, d)
        np.testing.assert_array_equal(host(gk), C.load(host(cache), page, d, again, 0))
        np.testing.assert_array_equal(host(gv), C.load(host(cache), page, d, again, 1))
    assert cat.cat_device_status()[0] == 0


def test_read_into_given_tensors():
    cache = cat.cat_mx_cache(3, 2, 16, 64)
    k, v = torch.full((4, 2, 64), 7.0, device=DEV), torch.full((4, 2, 64), 7.0, device=DEV)
    gk, gv = cat.cat_mx_cache_read(cache, dev(np.arange(4, dtype=np.int32)), 64, k=k, v=v)
    assert gk is k and gv is v and not k.any() and not v.any()


def test_every_scale_and_tie():
    """Every scale that a float32 block can have, over every grid value and middle, as keys and as values."""
    points = np.concatenate([R.GRID, R.MIDDLE, R.MIDDLE * (1 - 2.0 ** -20), R.MIDDLE * (1 + 2.0 ** -20), [7.5, 7.999]])
    x = np.zeros((253, 1, 64))
    for e in range(253):
        x[e, 0, 0] = 4.0
        x[e, 0, 1:32] = points
        x[e, 0, 32] = -4.0
        x[e, 0, 33:64] = -points
        x[e] *= 2.0 ** (e - 127.0) if e else 2.0 ** -126
    x = host(dev(x, torch.float32))                                  # (what float32 holds of the smallest)
    cache = cat.cat_mx_cache(8, 1, 32, 64)
    slots = np.arange(253, dtype=np.int32)
    cat.cat_mx_cache_write(dev(x, torch.float32), dev(-x, torch.float32), dev(slots), cache)
    same_cache(host(cache), C.store(C.blank(8, 1, 32, 64), 32, x, -x, slots), 32, 64)


def test_values_that_are_not_finite():
    x = np.ones((3, 2, 128))
    x[0, 0, 5], x[1, 1, 64], x[2, 0, 127] = np.inf, np.nan, -np.inf
    cache = cat.cat_mx_cache(1, 2, 16, 128)
    slots = np.arange(3, dtype=np.int32)
    cat.cat_mx_cache_write(dev(x, torch.bfloat16), dev(np.ones_like(x), torch.bfloat16), dev(slots), cache)
    assert cat.cat_device_status()[0] == 4
    same_cache(host(cache), C.store(C.blank(1, 2, 16, 128), 16, x, np.ones_like(x), slots), 16, 128)
    k, v = cat.cat_mx_cache_read(cache, dev(slots), 128)
    assert torch.isnan(k[0, 0, :32]).all() and torch.isfinite(k[0, 0, 32:]).all() and torch.isfinite(v).all()
    assert cat.cat_device_status()[0] == 0


def rope_case(rng, n, hq, hkv, d, page, dtype, rot, q_norm, k_norm, weight_dtype, table_rows=500):
    qkv = dev(heads(rng, n, hq + 2 * hkv, d).reshape(n, -1), TYPES[dtype])
    pages = -(-n // page) + 2
    a = np.arange(table_rows)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    cos, sin = dev(np.cos(a), torch.float32), dev(np.sin(a), torch.float32)
    pos = rng.integers(0, table_rows, n).astype(np.int32)
    pos[0] = 0
    wq = dev(1 + 0.2 * rng.standard_normal(d), TYPES[weight_dtype]) if q_norm else None
    wk = dev(1 + 0.2 * rng.standard_normal(d), TYPES[weight_dtype]) if k_norm else None
    return qkv, pages, cos, sin, pos, wq, wk


def rope_want(qkv, d, hq, hkv, pos, cos, sin, wq, wk, eps, interleaved):
    x = host(qkv).reshape(len(pos), -1, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    c, s = host(cos)[pos], host(sin)[pos]
    q = C.normed(q, None if wq is None else host(wq), eps)
    k = C.normed(k, None if wk is None else host(wk), eps)
    size = C.turned(np.abs(q), np.abs(c), -np.abs(s), interleaved), C.turned(np.abs(q), np.abs(c), np.abs(s), interleaved)
    return C.turned(q, c, s, interleaved), C.turned(k, c, s, interleaved), v, np.maximum(*size)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,hq,hkv,d,page,rot,interleaved,q_norm,k_norm,weights", [
    (1, 32, 8, 128, 64, 128, False, True, True, "bf16"), (1, 1, 1, 64, 16, 64, False, True, True, "f32"),
    (3, 5, 1, 256, 16, 256, False, True, True, "f32"), (9, 12, 12, 64, 16, 32, False, False, False, "f32"),
    (33, 7, 3, 64, 32, 64, True, True, False, "bf16"), (40, 4, 2, 128, 128, 64, False, False, True, "f32"),
    (17, 16, 4, 128, 64, 96, False, True, True, "bf16"), (21, 6, 2, 256, 64, 128, False, True, True, "bf16"),
    (50, 3, 1, 256, 32, 16, True, False, True, "f32"), (19, 2, 2, 128, 16, 48, True, True, True, "f32"),
    (65, 9, 1, 64, 64, 16, False, True, True, "bf16"), (300, 8, 2, 128, 64, 128, True, True, True, "bf16"),
])
def test_rope(n, hq, hkv, d, page, rot, interleaved, q_norm, k_norm, weights, dtype):
    rng = np.random.default_rng(n * d + rot)
    qkv, pages, cos, sin, pos, wq, wk = rope_case(rng, n, hq, hkv, d, page, dtype, rot, q_norm, k_norm, weights)
    slots = some_slots(rng, n, pages * page)
    cache = dev(C.blank(pages, hkv, page, d, 0x5A))
    before = host(cache)
    got = cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, q_weight=wq, k_weight=wk, eps=1e-5,
                                      interleaved=interleaved)
    q, k, v, size = rope_want(qkv, d, hq, hkv, pos, cos, sin, wq, wk, 1e-5, interleaved)
    assert got.dtype is torch.bfloat16 and got.shape == (n, hq, d)
    assert np.all(np.abs(host(got) - q) <= 20 * 2.0 ** -24 * size * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(q))
    same_cache(host(cache), C.store(before, page, k, v, slots), page, d)
    assert cat.cat_device_status()[0] == 0


def test_rope_keys_next_to_borders():
    """Keys whose exact values are at, and one float32 unit beside, middles of the grid and powers of two: turned by nothing, by a
    right angle, and by an angle whose products only float64 resolves."""
    d, page = 64, 16
    points = np.concatenate([R.MIDDLE, R.MIDDLE * (1 + 2.0 ** -23), R.MIDDLE * (1 - 2.0 ** -23), [4, 4 * (1 - 2.0 ** -24), 0, 3e-9]])
    n = 96
    rng = np.random.default_rng(3)
    x = rng.choice(np.concatenate([points, -points]), size=(n, 3, d))
    x[::3, :, 0] = 8 * (1 - 2.0 ** -24)
    x[1::3, :, 40] = 4.0
    qkv = dev(x.reshape(n, -1), torch.float32)
    a = np.array([0.0, np.pi / 2, 0.7, 2.0 ** -13])
    cos, sin = np.repeat(np.cos(a)[:, None], d // 2, 1), np.repeat(np.sin(a)[:, None], d // 2, 1)
    cos[1], sin[1] = 0.0, 1.0
    cos, sin = dev(cos, torch.float32), dev(sin, torch.float32)
    pos = (np.arange(n) % 4).astype(np.int32)
    slots = np.arange(n, dtype=np.int32)
    for interleaved in (False, True):
        cache = cat.cat_mx_cache(n // page, 1, page, d)
        cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, interleaved=interleaved)
        _, k, v, _ = rope_want(qkv, d, 1, 1, pos, cos, sin, None, None, 0.0, interleaved)
        same_cache(host(cache), C.store(C.blank(n // page, 1, page, d), page, k, v, slots), page, d)


@pytest.mark.parametrize("dtype,norm,interleaved", [("bf16", True, False), ("f32", True, True), ("f32", False, False), ("bf16", False, True)])
def test_rope_many_keys(dtype, norm, interleaved):
    """Some millions of keys, of which float32 would round some hundreds otherwise than their exact values."""
    n, hkv, d, page = 6000, 4, 128, 64
    rng = np.random.default_rng(11)
    qkv, pages, cos, sin, pos, _, wk = rope_case(rng, n, 1, hkv, d, page, dtype, d, False, norm, "f32")
    slots = np.arange(n, dtype=np.int32)
    cache = cat.cat_mx_cache(pages, hkv, page, d)
    cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, k_weight=wk, interleaved=interleaved)
    x = host(qkv).reshape(n, -1, d)[:, 1:1 + hkv]
    k = C.turned(C.normed(x, None if wk is None else host(wk), 1e-6), host(cos)[pos], host(sin)[pos], interleaved)
    codes, b = R.quantize(k.reshape(-1, d))
    got, _ = cat.cat_mx_cache_read(cache, dev(slots), d)
    np.testing.assert_array_equal(host(got).reshape(-1, d), R.values(codes, b))


@pytest.mark.parametrize("size", [1e-30, 1e-15, 1e15, 1e30])
def test_rope_rows_whose_squares_leave_float32(size):
    n, hq, hkv, d, page = 6, 2, 1, 128, 16
    rng = np.random.default_rng(5)
    qkv, pages, cos, sin, pos, wq, wk = rope_case(rng, n, hq, hkv, d, page, "f32", d, True, True, "f32")
    qkv = qkv * float(size)
    qkv[1] = 1.0                                                     # (no row of zeros without an eps)
    qkv[2, :] += 0.5 * float(size)
    slots = np.arange(n, dtype=np.int32)
    cache = cat.cat_mx_cache(pages, hkv, page, d)
    got = cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, q_weight=wq, k_weight=wk, eps=0.0)
    q, k, v, m = rope_want(qkv, d, hq, hkv, pos, cos, sin, wq, wk, 0.0, False)
    assert np.all(np.abs(host(got) - q) <= 20 * 2.0 ** -24 * m * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(q))
    same_cache(host(cache), C.store(C.blank(pages, hkv, page, d), page, k, v, slots), page, d)


def test_rope_positions_outside_the_tables():
    n, hq, hkv, d, page = 4, 3, 2, 64, 16
    rng = np.random.default_rng(6)
    qkv, pages, cos, sin, pos, wq, wk = rope_case(rng, n, hq, hkv, d, page, "bf16", d, True, True, "f32")
    pos[1], pos[2] = -1, 500
    slots = np.arange(n, dtype=np.int32)
    cache = cat.cat_mx_cache(pages, hkv, page, d)
    got = cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), cache, q_weight=wq, k_weight=wk)
    assert cat.cat_device_status()[0] == 4
    assert torch.isnan(got[1:3]).all() and torch.isfinite(got[0]).all() and torch.isfinite(got[3]).all()
    k, v = cat.cat_mx_cache_read(cache, dev(slots), d)
    assert torch.isnan(k[1:3]).all() and torch.isfinite(k[0]).all() and torch.isfinite(v).all()


def test_rope_equals_its_parts():
    """Values of a fused pass are cat_mx_cache_write's, whatever the batch."""
    n, hq, hkv, d, page = 70, 4, 2, 128, 32
    rng = np.random.default_rng(8)
    qkv, pages, cos, sin, pos, wq, wk = rope_case(rng, n, hq, hkv, d, page, "bf16", d, True, True, "bf16")
    slots = rng.permutation(pages * page)[:n].astype(np.int32)
    whole, single = cat.cat_mx_cache(pages, hkv, page, d), cat.cat_mx_cache(pages, hkv, page, d)
    q = cat.cat_mx_rope_cache_write(qkv, d, dev(pos), cos, sin, dev(slots), whole, q_weight=wq, k_weight=wk)
    for i in range(n):
        one = cat.cat_mx_rope_cache_write(qkv[i:i + 1], d, dev(pos[i:i + 1]), cos, sin, dev(slots[i:i + 1]), single, q_weight=wq,
                                          k_weight=wk)
        assert torch.equal(one[0], q[i])
    assert torch.equal(whole, single)
    v = qkv.view(n, -1, d)[:, hq + hkv:].contiguous()
    other = cat.cat_mx_cache_write(v, v, dev(slots), cat.cat_mx_cache(pages, hkv, page, d))
    assert torch.equal(other[:, 1], whole[:, 1])


def test_streams_and_graphs():
    """A captured rotation and read, replayed with other tokens, positions and slots beside calls on another stream."""
    n, hq, hkv, d, page = 50, 4, 2, 128, 16
    rng = np.random.default_rng(12)
    qkv, pages, cos, sin, pos, wq, wk = rope_case(rng, n, hq, hkv, d, page, "bf16", d, True, True, "bf16")
    slots = rng.permutation(pages * page)[:n].astype(np.int32)
    other = rng.permutation(pages * page)[:n].astype(np.int32)
    cache, aside = cat.cat_mx_cache(pages, hkv, page, d), cat.cat_mx_cache(pages, hkv, page, d)
    x, p, s = qkv.clone(), dev(pos), dev(slots)
    run = lambda c: cat.cat_mx_rope_cache_write(x, d, p, cos, sin, s, c, q_weight=wq, k_weight=wk)  # noqa: E731
    run(cache)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q = run(cache)
        k, v = cat.cat_mx_cache_read(cache, s, d)
    x.copy_(qkv.flip(0))
    s.copy_(dev(other))
    cache.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            q2 = run(aside)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(cache, aside)
    wk_, wv_ = cat.cat_mx_cache_read(cache, s, d)
    assert torch.equal(k, wk_) and torch.equal(v, wv_)
    assert cat.cat_device_status()[0] == 0


def test_rows_of_a_large_cache():
    """Rows whose bytes lie behind 2^32 of the cache's first."""
    page, hkv, d = 1024, 8, 256
    pages = 4 * 2 ** 30 // (2 * hkv * C.page_bytes(page, d)) + 2
    cache = cat.cat_mx_cache(pages, hkv, page, d)
    rng = np.random.default_rng(13)
    k, v = heads(rng, 20, hkv, d), heads(rng, 20, hkv, d)
    slots = (pages * page - 1 - 7 * np.arange(20)).astype(np.int32)
    cat.cat_mx_cache_write(dev(k, torch.float32), dev(v, torch.float32), dev(slots), cache)
    gk, gv = cat.cat_mx_cache_read(cache, dev(slots), d)
    for got, x in ((gk, k), (gv, v)):
        np.testing.assert_array_equal(host(got).reshape(-1, d), R.values(*R.quantize(host(dev(x, torch.float32)).reshape(-1, d))))
    assert not cache[:pages - 1].any()
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV)
    q = torch.ones((2, hkv, d), dtype=torch.bfloat16, device=DEV)
    small = cache[pages - 1:].clone()
    for rows in (1, 2):
        off = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
        lens = torch.tensor([1024], dtype=torch.int32, device=DEV)
        far = cat.cat_mx_attention(q[:rows], cache, table, lens, 0.1, offsets=off)
        assert torch.equal(far, cat.cat_mx_attention(q[:rows], small, table * 0, lens, 0.1, offsets=off)) and bool(far.any())
