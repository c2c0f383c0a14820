"""The microscaled 4-bit operators on the GPU against float64.

Quantization of given values is exact arithmetic (a power-of-two scale, one rounding): every code and scale byte is
the reference's.  Behind a norm or SwiGLU the values carry float32 rounding: with eps_v the bound on their relative
error, a code may be the neighbour of the reference's only where the exact value / scale lies within eps_v (relative)
of the middle between the two, and blocks whose largest magnitude is within eps_v of a power of two are left out
(their scale may be either).  eps_v = 1e-5: a mean of d squares in float32 sums is within 1e-6 (partial sums of at most
d / 256 + 10 terms), a square root, a division and three products add 4e-7; SwiGLU's exponential is within
(2 + 1.2 |g|) 2^-23, 3e-6 at |g| = 20.
Products: codes' products are exact and summed in float32 in some order, each addition within 2^-23 of the sum of
magnitudes so far (truncation included): |y - y64| <= d 2^-23 sum |x w|, plus half a unit of bfloat16
(its significand has 8 bits: 2^-8 |y|) where the output has 16 bits."""
import numpy as np
import pytest
import torch

import mx_reference as R

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")
DEV = "cuda"
EPS_V = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.detach().double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def tokens(rng, n, d):
    """Rows with outlier channels, small rows, a zero row and a zero block."""
    x = rng.standard_normal((n, d)) * np.exp(rng.standard_normal((n, 1)))
    x[:, rng.choice(d, max(1, d // 50), replace=False)] *= 100.0
    if n > 2:
        x[1] = 0.0
        x[2, :32] = 0.0
    return x


def poisoned(n, d):
    return (torch.full((n, d // 2), 0xA5, dtype=torch.uint8, device=DEV),
            torch.full((n, R.pitch(d)), 0xA5, dtype=torch.uint8, device=DEV))


def same_form(xq, xs, codes, b):
    q, s = R.pack(codes, b)
    np.testing.assert_array_equal(xs.cpu().numpy(), s)              # the pad bytes are zeros too
    got = xq.cpu().numpy()
    # a value that rounds to zero may keep its sign: codes 0 and 8 are the same value
    np.testing.assert_array_equal(R.values(*R.unpack(got, s)), R.values(codes, b))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 32), (3, 64), (5, 96), (1, 4096), (7, 480), (9, 512), (33, 544), (130, 1120),
                                 (257, 256), (1000, 4096), (2, 14336), (3, 262144)])
def test_quantize(n, d, dtype):
    x = dev(tokens(np.random.default_rng(n * d), n, d), TYPES[dtype])
    xq, xs = cat.cat_mx_quantize(x, xq=poisoned(n, d)[0], xs=poisoned(n, d)[1])
    codes, b = R.quantize(host(x))
    same_form(xq, xs, codes, b)
    for out in TYPES.values():
        np.testing.assert_array_equal(host(cat.cat_mx_dequantize(xq, xs, out_dtype=out)), R.values(codes, b))
    assert cat.cat_device_status()[0] == 0


def test_quantize_every_tie_and_scale():
    """Every grid value, middle and neighbour of a middle under every scale that a float32 block can have."""
    points = np.concatenate([R.GRID, R.MIDDLE, R.MIDDLE * (1 - 2.0 ** -20), R.MIDDLE * (1 + 2.0 ** -20), [7.5, 7.999]])
    points = np.concatenate([points, -points])
    rows = np.zeros((254, 64))
    with np.errstate(over="ignore"):
        for e in range(254):
            rows[e, :32] = 0.0
            rows[e, 0] = 4.0
            rows[e, 1:32] = points[:31]
            rows[e, 32] = -7.0
            rows[e, 33:64] = points[-31:]
            rows[e] *= 2.0 ** (e - 129)
    x = rows.astype(np.float32)
    assert np.isfinite(x).all()
    xd = dev(x)
    xq, xs = cat.cat_mx_quantize(xd)
    same_form(xq, xs, *R.quantize(x.astype(np.float64)))


def test_quantize_what_is_not_finite():
    x = np.random.default_rng(5).standard_normal((6, 128))
    x[0, 3], x[1, 40], x[2, 127], x[3, 0] = np.nan, np.inf, -np.inf, 3.4e38
    for dtype in TYPES.values():
        xd = dev(x, dtype)
        xq, xs = cat.cat_mx_quantize(xd)
        same_form(xq, xs, *R.quantize(host(xd)))
        v = host(cat.cat_mx_dequantize(xq, xs))
        assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:64]).all() and np.isnan(v[2, 96:]).all()
        given = np.isfinite(host(xd).reshape(6, 4, 32)).all(-1).repeat(32, -1)   # (3.4e38 is an infinity in bfloat16)
        np.testing.assert_array_equal(np.isfinite(v), given)
        st, word = cat.cat_device_status()
        assert st == 4 and word & 2
    assert cat.cat_device_status()[0] == 0


def test_quantize_gathered_rows():
    rng = np.random.default_rng(6)
    x = tokens(rng, 50, 352)
    rows = rng.integers(0, 50, 133).astype(np.int32)
    rows[[0, 7, 9]] = [-1, 50, 2 ** 31 - 1]                         # outside: rows of zeros
    xd = dev(x, torch.bfloat16)
    xq, xs = cat.cat_mx_quantize(xd, rows=dev(rows))
    padded = np.concatenate([host(xd), np.zeros((1, 352))])
    same_form(xq, xs, *R.quantize(padded[np.where((rows < 0) | (rows >= 50), 50, rows)]))
    none = torch.empty((0, 352), dtype=torch.bfloat16, device=DEV)
    assert not cat.cat_mx_quantize(none, rows=dev(rows))[0].any()   # no row to take
    assert cat.cat_mx_quantize(none)[0].shape == (0, 176)
    assert cat.cat_device_status()[0] == 0


def near(xq, xs, v):
    """The 4-bit form of values known to EPS_V against float64 v: see above."""
    codes, b = R.quantize(v)
    got, gb = R.unpack(xq.cpu().numpy(), xs.cpu().numpy())
    a = np.abs(v.reshape(*b.shape, 32)).max(-1)
    m, _ = np.frexp(a)
    sure = (b > 0) & (m < 1 - EPS_V) & (m > 0.5 * (1 + EPS_V)) | (a == 0)
    np.testing.assert_array_equal(gb[sure], b[sure])
    assert sure.mean() > 0.99
    scaled = np.abs(v) / np.exp2(b - 127.0).repeat(32, -1)
    at = sure.repeat(32, -1) & (R.values(got, gb) != R.values(codes, b))
    assert at.mean() < 1e-3
    lower = np.minimum(got & 7, codes & 7)[at]
    assert np.all(np.abs((got & 7) - (codes & 7))[at] == 1)
    assert np.all(np.abs(scaled[at] / R.MIDDLE[lower] - 1) <= EPS_V)
    assert np.all((scaled[at] < 0.26) | ((got >> 3) == (codes >> 3))[at])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 32), (4, 96), (27, 4096), (300, 544), (65, 1120), (5, 9024), (3, 14336), (2, 40000),
                                 (2, 262144)])
def test_swiglu(n, d, dtype):
    rng = np.random.default_rng(n + d)
    gu = rng.standard_normal((n, 2 * d)) * 4
    gu[0, :4] = [-100.0, 100.0, 0.0, 19.0]
    g = dev(gu, TYPES[dtype])
    v = host(g)
    v = v[:, :d] / (1 + np.exp(-v[:, :d])) * v[:, d:]
    near(*cat.cat_mx_swiglu_quantize(g), v)
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("dtype,weight", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,d", [(1, 32), (4, 96), (27, 4096), (300, 544), (65, 1120), (5, 9024), (3, 14336), (2, 40000),
                                 (2, 262144), (20000, 64)])
def test_rmsnorm(n, d, dtype, weight):
    rng = np.random.default_rng(n + d)
    x, r = dev(tokens(rng, n, d), TYPES[dtype]), dev(3 * rng.standard_normal((n, d)), TYPES[dtype])
    if n > 2:
        r[1] = 0.0                                                  # a row of zeros
    w = dev(1 + 0.2 * rng.standard_normal(d), TYPES[weight])
    for res in (r, None):
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=res)
        total = host(x) + (host(r) if res is not None else 0.0)
        exact = x.float() + r.float() if res is not None else x
        assert torch.equal(h, exact.to(x.dtype))
        v = total / np.sqrt((total ** 2).mean(-1, keepdims=True) + 1e-5) * host(w)
        near(xq, xs, v)
    # the sum over x or over the residual
    for where in (0, 1):
        pair = [x.clone(), r.clone()]
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(pair[0], w, 1e-5, residual=pair[1], h=pair[where])
        first = cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=r)
        assert h is pair[where] and all(torch.equal(a, b) for a, b in zip((xq, xs, h), first))
        assert torch.equal(pair[1 - where], (x, r)[1 - where])
    assert cat.cat_device_status()[0] == 0


def test_rmsnorm_of_rows_that_are_not_finite_or_zero():
    x = torch.randn(5, 256, device=DEV)
    x[0, 3], x[1, 200], x[2] = float("nan"), float("inf"), 0.0
    w = torch.ones(256, device=DEV)
    xq, xs, _ = cat.cat_mx_rmsnorm_quantize(x, w, 0.0, residual=torch.zeros_like(x))
    v = cat.cat_mx_dequantize(xq, xs)
    assert torch.isnan(v[0]).all()
    assert torch.isnan(v[1, 192:224]).all()                          # inf / inf; the others are 0 / 1
    assert torch.isfinite(v[3:]).all() and v[3:].abs().max() > 0
    assert cat.cat_device_status()[0] == 4
    xq, xs, _ = cat.cat_mx_rmsnorm_quantize(x, w, 1e-6, residual=torch.zeros_like(x))
    assert not cat.cat_mx_dequantize(xq, xs)[2].any()                # a row of zeros stays one
    cat.cat_device_status()


def operand(rng, rows, d, spread=0.5):
    """A random matrix in the 4-bit form: all codes, scales of unequal size; zero rows and blocks among them."""
    codes = rng.integers(0, 16, (rows, d))
    b = np.clip(np.round(127 + rng.standard_normal((rows, d // 32)) * spread), 120, 134).astype(np.int64)
    if rows > 3:
        codes[1] = 0
        codes[2, :32] = 8
    q, s = R.pack(codes, b)
    s[:, d // 32:] = 255                                            # the pad bytes' values must not matter
    return dev(q), dev(s), dev(R.values(codes, b))


def check_product(y, x, w):
    ref = x @ w.T
    bound = x.shape[1] * 2.0 ** -23 * (x.abs() @ w.abs().T) + 1e-30
    if y.dtype is torch.bfloat16:
        bound = bound + 2.0 ** -8 * ref.abs()
    assert bool(((y.double() - ref).abs() <= bound).all()), float(((y.double() - ref).abs() / bound).max())


SHAPES = [(1, 32, 1), (1, 32, 128), (2, 64, 5), (1, 4096, 6144), (7, 96, 129), (8, 512, 256), (9, 544, 300), (16, 4096, 1000),
          (17, 1024, 8), (27, 14336, 512), (33, 1120, 257), (64, 256, 640), (65, 2048, 130), (100, 4096, 384), (129, 736, 511),
          (200, 8192, 128), (201, 4096, 6144), (257, 512, 1000), (300, 1056, 2049), (511, 4064, 4096), (512, 2080, 4097),
          (1000, 256, 256), (1025, 1120, 1173), (2048, 4096, 6144), (3001, 544, 3000)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,d_out", SHAPES)
def test_linear(n, d, d_out, out):
    rng = np.random.default_rng(n + d + d_out)
    xq, xs, x = operand(rng, n, d)
    wq, ws, w = operand(rng, d_out, d)
    guard = torch.full((n * d_out + 512,), -7.0, dtype=TYPES[out], device=DEV)
    y = guard[256:256 + n * d_out].view(n, d_out)                   # nothing before or behind it is written
    y.fill_(float("nan"))
    cat.cat_mx_linear(xq, xs, wq, ws, y=y)
    check_product(y, x, w)
    assert bool((guard[:256] == -7).all()) and bool((guard[256 + n * d_out:] == -7).all())
    assert torch.equal(cat.cat_mx_linear(xq, xs, wq, ws, out_dtype=TYPES[out]), y)     # the same each time
    assert cat.cat_device_status()[0] == 0


def test_linear_of_no_tokens():
    rng = np.random.default_rng(1)
    wq, ws, _ = operand(rng, 64, 128)
    xq, xs = (torch.empty((0, b), dtype=torch.uint8, device=DEV) for b in (64, 16))
    assert cat.cat_mx_linear(xq, xs, wq, ws).shape == (0, 64)


@pytest.mark.parametrize("n,d,d_out", [(3, 256, 200), (40, 1024, 300), (700, 512, 700)])
def test_linear_scales_from_end_to_end(n, d, d_out):
    """Scales far from 1 on either side, and NaN scales: only the outputs that use them are NaN."""
    rng = np.random.default_rng(d)
    codes = [rng.integers(0, 16, (r, d)) for r in (n, d_out)]
    b = [np.full((r, d // 32), base, dtype=np.int64) + rng.integers(-3, 4, (r, d // 32)) for r, base in ((n, 200), (d_out, 60))]
    b[0][1, 3] = b[1][5, 0] = b[1][d_out - 1, d // 32 - 1] = 255
    (xq, xs), (wq, ws) = (tuple(dev(t) for t in R.pack(c, s)) for c, s in zip(codes, b))
    x, w = (dev(R.values(c, s)) for c, s in zip(codes, b))
    y = cat.cat_mx_linear(xq, xs, wq, ws)
    bad = torch.zeros((n, d_out), dtype=torch.bool, device=DEV)
    bad[1] = True
    bad[:, 5] = True
    bad[:, d_out - 1] = True
    assert torch.equal(torch.isnan(y), bad)
    x, w = x.nan_to_num(0.0), w.nan_to_num(0.0)
    check_product(torch.where(bad, (x @ w.T).float(), y), x, w)


GROUPS = [
    ([1], 64, 40), ([0, 1, 0], 512, 300), ([3, 0, 5, 1, 0, 0, 7], 1024, 256), ([16, 16], 4096, 1000), ([129, 0, 255, 40], 544, 500),
    ([300, 1, 700, 0, 33], 1120, 700), ([1] * 64, 256, 96), ([0] * 9, 128, 64), ([5] * 500, 64, 33), ([1500, 9, 600, 100], 2048, 1024),
    ([700, 650, 0, 900, 801], 256, 2000), ([2, 30] * 20, 2080, 513),
]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d,d_out", GROUPS, ids=lambda v: str(sum(v)) + "in" + str(len(v)) if isinstance(v, list) else str(v))
@pytest.mark.parametrize("before,behind", [(0, 0), (3, 130)])
def test_grouped(counts, d, d_out, before, behind, out):
    rng = np.random.default_rng(sum(counts) + d)
    experts, m = len(counts), before + sum(counts) + behind
    edges = before + np.concatenate([[0], np.cumsum(counts)])
    xq, xs, x = operand(rng, m, d)
    wq, ws, w = operand(rng, experts * d_out, d)
    w = w.view(experts, d_out, d)
    guard = torch.full((m * d_out + 512,), -7.0, dtype=TYPES[out], device=DEV)
    y = guard[256:256 + m * d_out].view(m, d_out)
    y.fill_(float("nan"))
    cat.cat_mx_linear_grouped(xq, xs, wq.view(experts, d_out, -1), ws.view(experts, d_out, -1), dev(edges.astype(np.int32)), y=y)
    for e in range(experts):
        if counts[e]:
            check_product(y[edges[e]:edges[e + 1]], x[edges[e]:edges[e + 1]], w[e])
    assert not y[:before].any() and not y[before + sum(counts):].any()   # (a NaN counts as true)
    assert bool((guard[:256] == -7).all()) and bool((guard[256 + m * d_out:] == -7).all())
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("given,taken", [
    ([-5, 40, 100], [0, 40, 64]), ([10, 5, 60], [10, 10, 60]), ([64, 64, 64], [64, 64, 64]), ([0, 2 ** 31 - 1, 3], [0, 64, 64]),
    ([-2 ** 31, -1, 64], [0, 0, 64]),
])
def test_grouped_offsets_out_of_order_or_range(given, taken):
    rng = np.random.default_rng(3)
    xq, xs, x = operand(rng, 64, 256)
    wq, ws, w = operand(rng, 2 * 150, 256)
    w = w.view(2, 150, 256)
    y = cat.cat_mx_linear_grouped(xq, xs, wq.view(2, 150, -1), ws.view(2, 150, -1), dev(np.array(given, dtype=np.int32)))
    rest = torch.ones(64, dtype=torch.bool, device=DEV)
    for e in range(2):
        if taken[e + 1] > taken[e]:
            check_product(y[taken[e]:taken[e + 1]], x[taken[e]:taken[e + 1]], w[e])
        rest[taken[e]:taken[e + 1]] = False
    assert not y[rest].any()


def test_grouped_is_the_linear_of_each_group():
    """One expert with all rows is the plain product, bit for bit where both cut their sums the same way."""
    rng = np.random.default_rng(4)
    xq, xs, x = operand(rng, 90, 512)
    wq, ws, w = operand(rng, 200, 512)
    y = cat.cat_mx_linear_grouped(xq, xs, wq[None], ws[None], dev(np.array([0, 90], dtype=np.int32)))
    check_product(y, x, w)


def nan_rows(s, rows):
    s = s.clone()
    s[rows] = 255
    return s


@pytest.mark.parametrize("counts,d,d_out", [([3, 0, 5, 1], 512, 200), ([300, 20, 500], 1056, 384)])
def test_grouped_products_use_their_own_rows_alone(counts, d, d_out):
    """NaN scales in all of the other experts' rows and weights, and in the rows of no group, do not reach a group."""
    rng = np.random.default_rng(11)
    m = sum(counts) + 9
    edges = 4 + np.concatenate([[0], np.cumsum(counts)])
    xq, xs, x = operand(rng, m, d)
    wq, ws, w = operand(rng, len(counts) * d_out, d)
    w, wq, ws = (t.view(len(counts), d_out, -1) for t in (w, wq, ws))
    for e in range(len(counts)):
        mine = slice(edges[e], edges[e + 1])
        others = torch.ones(m, dtype=torch.bool, device=DEV)
        others[mine] = False
        other_w = torch.arange(len(counts), device=DEV) != e
        y = cat.cat_mx_linear_grouped(xq, nan_rows(xs, others), wq, nan_rows(ws, other_w), dev(edges.astype(np.int32)))
        if counts[e]:
            check_product(y[mine], x[mine], w[e])
        assert not y[:4].any() and not y[-5:].any()


def test_sizes_past_32_bits():
    """Outputs, values and codes whose element numbers and byte offsets need more than 32 bits: the last rows are right."""
    rng = np.random.default_rng(12)
    n, d, d_out = 70001, 64, 65536
    xq, xs, _ = operand(rng, n, d)
    wq, ws, w = operand(rng, d_out, d)
    y = cat.cat_mx_linear(xq, xs, wq, ws, out_dtype=torch.bfloat16)
    tail = slice(n - 40, n)
    check_product(y[tail], cat.cat_mx_dequantize(xq[tail].contiguous(), xs[tail].contiguous()).double(), w)
    grouped = cat.cat_mx_linear_grouped(xq, xs, wq[None], ws[None], dev(np.array([30, n - 20], dtype=np.int32)),
                                        out_dtype=torch.bfloat16)
    assert torch.equal(grouped[n - 40:n - 20], y[n - 40:n - 20]) and not grouped[n - 20:].any() and not grouped[:30].any()
    del y, grouped
    n, d = 140001, 32768
    x = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
    x[-2:] = torch.randn((2, d), device=DEV)
    xq, xs = cat.cat_mx_quantize(x)
    same_form(xq[-2:], xs[-2:], *R.quantize(host(x[-2:])))
    v = cat.cat_mx_dequantize(xq, xs, out_dtype=torch.bfloat16)
    assert torch.equal(v[-2:], cat.cat_mx_dequantize(xq[-2:].contiguous(), xs[-2:].contiguous(), out_dtype=torch.bfloat16))
    assert not v[:-2].any()
    del v
    hq, hs, h = cat.cat_mx_rmsnorm_quantize(x, torch.ones(d, device=DEV), 1e-5, residual=x)
    last = cat.cat_mx_rmsnorm_quantize(x[-2:].contiguous(), torch.ones(d, device=DEV), 1e-5, residual=x[-2:].contiguous())
    assert torch.equal(hq[-2:], last[0]) and torch.equal(hs[-2:], last[1]) and torch.equal(h[-2:], last[2])


@pytest.mark.parametrize("n,d,d_out", [(40, 131072, 1024), (16, 65536, 8192), (1000, 65536, 4096)],
                         ids=["split", "single", "pairs"])
def test_bounded_wait_gives_up_then_library_recovers(n, d, d_out):
    """Waits that run out (a bound of 1 ns): the kernel drains, returns and says so; the next call is right."""
    rng = np.random.default_rng(13)
    xq, xs, x = operand(rng, n, d)
    wq, ws, w = operand(rng, d_out, d)
    assert cat.cat_device_status()[0] == 0
    try:
        cat.cat_set_wait_limit_ns(1)
        cat.cat_mx_linear(xq, xs, wq, ws)
        st, word = cat.cat_device_status()
    finally:
        cat.cat_set_wait_limit_ns(0)
    assert st == 7 and word & 1 and word & 1 << 14 and word >> 16, hex(word)
    for _ in range(2):
        check_product(cat.cat_mx_linear(xq, xs, wq, ws), x, w)
    assert cat.cat_device_status()[0] == 0


def test_on_several_streams():
    """Calls of all kinds on streams of their own, at once."""
    rng = np.random.default_rng(8)
    calls = []
    for n, d, d_out in ((5, 2048, 1000), (40, 1024, 3000), (900, 1024, 900), (16, 4096, 2048)):
        xq, xs, x = operand(rng, n, d)
        wq, ws, w = operand(rng, d_out, d)
        calls.append((torch.cuda.Stream(), (xq, xs, wq, ws), torch.empty(n, d_out, device=DEV), x, w))
    torch.cuda.synchronize()
    for _ in range(10):
        for stream, args, y, _, _ in calls:
            with torch.cuda.stream(stream):
                y.fill_(float("nan"))
                cat.cat_mx_linear(*args, y=y)
    torch.cuda.synchronize()
    for _, _, y, x, w in calls:
        check_product(y, x, w)
    assert cat.cat_device_status()[0] == 0


def test_in_a_graph():
    """A layer with experts captured once and replayed on other tokens."""
    rng = np.random.default_rng(9)
    x, r = (torch.randn(24, 512, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    gain = torch.ones(512, device=DEV, dtype=torch.bfloat16)
    wq, ws, w = operand(rng, 4 * 256, 512)
    wq, ws = wq.view(4, 256, -1), ws.view(4, 256, -1)
    offsets = dev(np.array([0, 7, 7, 20, 24], dtype=np.int32))

    def layer():
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, gain, 1e-5, residual=r)
        y = cat.cat_mx_linear_grouped(xq, xs, wq, ws, offsets)
        return h, y, cat.cat_mx_linear(*cat.cat_mx_swiglu_quantize(y), wq[0, :, :64].contiguous(),
                                       ws[0, :, :16].contiguous())
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    for seed in range(3):
        torch.manual_seed(seed)
        x.normal_()
        offsets.copy_(dev(np.array([[0, 7, 7, 20, 24], [0, 0, 0, 0, 24], [2, 3, 9, 9, 20]][seed], dtype=np.int32)))
        graph.replay()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, layer()))


def test_refuses_other_tensors():
    x = torch.randn(8, 128, device=DEV)
    xq, xs = cat.cat_mx_quantize(x)
    wq, ws = cat.cat_mx_quantize(torch.randn(16, 128, device=DEV))
    offsets = dev(np.array([0, 4, 8], dtype=np.int32))
    with pytest.raises(TypeError):
        cat.cat_mx_quantize(x.half())
    with pytest.raises(TypeError):
        cat.cat_mx_linear(xq, xs, wq, ws, y=torch.empty(8, 16, device=DEV, dtype=torch.float16), out_dtype=torch.float16)
    with pytest.raises(cat.CatError):
        cat.cat_mx_quantize(torch.randn(8, 48, device=DEV))
    for bad in (lambda: cat.cat_mx_quantize(x.T), lambda: cat.cat_mx_quantize(x.cpu()),
                lambda: cat.cat_mx_quantize(x, rows=torch.zeros(3, device=DEV)),
                lambda: cat.cat_mx_linear(xq, xs[:, :8], wq, ws), lambda: cat.cat_mx_linear(xq, xs, wq[:, :32].contiguous(), ws),
                lambda: cat.cat_mx_linear(xq, xs, wq, ws, y=torch.empty(8, 17, device=DEV)),
                lambda: cat.cat_mx_linear_grouped(xq, xs, wq.view(2, 8, -1), ws.view(2, 8, -1), offsets[:2]),
                lambda: cat.cat_mx_linear_grouped(xq, xs, wq.view(2, 8, -1), ws.view(2, 8, -1), offsets.long()),
                lambda: cat.cat_mx_rmsnorm_quantize(x, x[0], 1e-5, residual=x[:4]),
                lambda: cat.cat_mx_rmsnorm_quantize(x, x[:, 0].contiguous(), 1e-5),
                lambda: cat.cat_mx_swiglu_quantize(x[:, :127].contiguous())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(cat.CatError):
        cat.cat_mx_rmsnorm_quantize(x, x[0].contiguous(), -1.0)
    unaligned = torch.randn(8 * 128 + 1, device=DEV)[1:].view(8, 128)
    with pytest.raises(cat.CatError):
        cat.cat_mx_quantize(unaligned)


@pytest.mark.parametrize("tokens,width,hidden,experts,top", [(1, 256, 512, 4, 2), (37, 1024, 1408, 8, 2), (600, 512, 256, 16, 4)])
def test_experts_example(tokens, width, hidden, experts, top):
    """A block's experts from the norm to the sum: the 4-bit block, stage by stage in float64 on its own codes, and its
    distance from float32.  Each product has quantization noise on both operands: 32 normal values on a grid whose step is
    1/4 to 1/8 of their largest have a relative error of about 0.11, sqrt(2) of that a product, and a second pair behind
    SwiGLU: 13 to 16 dB; 10 is asked for."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import mx_experts as E
    g = torch.Generator(device=DEV)
    g.manual_seed(tokens)
    randn = lambda *s, scale=1.0: (scale * torch.randn(*s, generator=g, device=DEV)).bfloat16()  # noqa: E731
    gain, router = 1 + randn(width, scale=0.1), randn(experts, width, scale=width ** -0.5)
    gate_up, down = randn(experts, 2 * hidden, width, scale=width ** -0.5), randn(experts, width, hidden, scale=hidden ** -0.5)
    x, r = randn(tokens, width), randn(tokens, width)
    block = E.Experts(gain, router, gate_up, down, top)
    y, (rows, offsets, shares) = block(x, r)
    assert offsets[-1] == tokens * top and torch.equal(torch.bincount(rows.long(), minlength=tokens).cpu(), torch.full((tokens,), top))
    xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, gain, 1e-5, residual=r)
    v = cat.cat_mx_dequantize(xq, xs).double()[rows.long()]
    want = h.double()
    values = lambda w: cat.cat_mx_dequantize(w[0].flatten(0, 1), w[1].flatten(0, 1)).double().view(*w[0].shape[:2], -1)  # noqa: E731
    wg, wd = values(block.gate_up), values(block.down)
    edges = offsets.tolist()
    gu = torch.cat([v[a:b] @ wg[e].T for e, (a, b) in enumerate(zip(edges, edges[1:]))]).to(torch.bfloat16)
    act = cat.cat_mx_dequantize(*cat.cat_mx_swiglu_quantize(gu.contiguous())).double()
    out = torch.cat([act[a:b] @ wd[e].T for e, (a, b) in enumerate(zip(edges, edges[1:]))])
    want.index_add_(0, rows.long(), out * shares.double()[:, None])
    # (a gate or u whose bf16 rounding differs moves a code of the next operand now and then)
    assert float((y.double() - want).norm() / want.norm()) < 1e-2
    _, _, _, db = E.run(tokens, width, hidden, experts, top)
    assert db > 10.0 and cat.cat_device_status()[0] == 0
