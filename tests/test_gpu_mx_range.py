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
