"""The microscaled norm and SwiGLU at the ends of float32's range, against float64.

The bounds are those of the ordinary values (EPS_V = 1e-5 on a value before its one rounding to 4 bits, see
test_gpu_mx.py): the inputs here are such that float32 can hold every step of the stated formulas to that."""
import numpy as np
import pytest
import torch

import mx_reference as R
from test_gpu_mx import TYPES, cat, dev, host, near

pytestmark = pytest.mark.gpu


def signs(rng, shape):
    return np.where(rng.random(shape) < 0.5, -1.0, 1.0)


def test_swiglu_of_gates_below_the_smallest_normal_number():
    """Gates of 2 j units of 2^-149, j of 1 to 4095, with u of about 2^120: silu(g) = g / 2 is exactly j units, the
    product an ordinary number known to float32's rounding."""
    rng = np.random.default_rng(21)
    rows, d = 12, 256
    j = np.stack([rng.integers(1 << i, 2 << i, d) for i in range(rows)])
    g = signs(rng, (rows, d)) * j * 2.0 ** -148
    u = signs(rng, (rows, d)) * rng.uniform(1.0, 2.0, (rows, d)) * 2.0 ** 120
    gu = dev(np.concatenate([g, u], 1), torch.float32)
    held = host(gu)
    assert np.array_equal(held[:, :d], g)
    near(*cat.cat_mx_swiglu_quantize(gu), held[:, :d] / (1 + np.exp(-held[:, :d])) * held[:, d:])
    assert cat.cat_device_status()[0] == 0


# a row kernel each: a warp, a CTA with one and with two halves a thread, two readings
WIDTHS = [96, 512, 4096, 9024, 14336, 40000]


def check_norm(x, r, w, eps):
    """The norm with the residual against float64: the sum exactly, the 4-bit form as near as `near` asks."""
    for res in (r, None):
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, w, eps, residual=res)
        total = host(x) + (host(res) if res is not None else 0.0)
        assert torch.equal(h, (x.float() + res.float()).to(x.dtype) if res is not None else x)
        near(xq, xs, total / np.sqrt((total ** 2).mean(-1, keepdims=True) + eps) * host(w))
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,gain,eps", [(1e15, 1e30, 1e-5), (1e-15, 1e-30, 1e-35)])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_whose_gain_and_values_leave_the_range_together(d, size, gain, eps, dtype):
    """Values times gain would overflow or vanish; the normalized value times gain is an ordinary number."""
    rng = np.random.default_rng(d)
    x, r = (dev(size * rng.standard_normal((5, d)), TYPES[dtype]) for _ in range(2))
    check_norm(x, r, dev(gain * (1 + 0.2 * rng.standard_normal(d)), TYPES[dtype]), eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,eps", [(1e20, 1e-5), (1e28, 0.0), (1e37, 1e-5), (1e-21, 0.0), (1e-30, 0.0), (1e-22, 2.0 ** -149)])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_whose_squares_leave_the_range(d, size, eps, dtype):
    """Squares overflow or vanish, the norm does not: rows of such values beside an ordinary row."""
    rng = np.random.default_rng(d + 1)
    rows = np.array([size, 1.0, size, 3 * size, size])[:, None]
    x, r = (dev(rows * rng.standard_normal((5, d)), TYPES[dtype]) for _ in range(2))
    check_norm(x, r, dev(1 + 0.2 * rng.standard_normal(d), TYPES[dtype]), eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_of_the_largest_numbers(d, dtype):
    """Every value the largest of its type: the normalized ones are 1."""
    largest = torch.finfo(TYPES[dtype]).max
    x = torch.full((3, d), largest, dtype=TYPES[dtype], device="cuda")
    x[1, ::2] = -largest
    xq, xs, _ = cat.cat_mx_rmsnorm_quantize(x, torch.full((d,), 1.01, device="cuda"), 1e-5)
    v = cat.cat_mx_dequantize(xq, xs)
    assert torch.equal(v, torch.sign(x.float()))                    # 1.01 is nearest to 1
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("d", WIDTHS)
def test_norm_of_an_infinity_beside_rows_out_of_range(d):
    """A row with an infinity still says so, with NaN in its block and zeros elsewhere; rows of zeros with eps = 0 are NaN."""
    x = torch.full((4, d), 1e25, device="cuda")
    x[1, 40] = float("inf")
    x[2] = 0.0
    xq, xs, _ = cat.cat_mx_rmsnorm_quantize(x, torch.ones(d, device="cuda"), 0.0)
    v = cat.cat_mx_dequantize(xq, xs)
    # 1 is a power of two: known to 1e-5, a block's largest value may be below it, under half the scale, and 6 / 8 the most there
    assert bool(((v[0] == 1.0) | (v[0] == 0.75)).all()) and torch.equal(v[3], v[0])
    assert torch.isnan(v[1, 32:64]).all() and not v[1, :32].any() and not v[1, 64:].any()
    assert torch.isnan(v[2]).all()
    assert cat.cat_device_status()[0] == 4
