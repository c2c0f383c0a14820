"""The microscaled 4-bit operators without a GPU: the reference's own grid, and what the library refuses."""
import ctypes

import numpy as np
import pytest

import mx_reference as R
import paper_2603_04359_gb300 as cat
from paper_2603_04359_gb300 import build as catbuild
from fake_runtime import FakeRuntime, ensure_built

P, BAD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    ensure_built()
    return cat.load_library()


def test_reference_rounds_to_the_nearest_grid_value():
    x = np.linspace(-8, 8, 32 * 512).reshape(-1, 32).copy()
    x[:, 0] = 4.0                                                  # every block's scale is 1
    x[:, 1:] = np.clip(x[:, 1:], -7.99, 7.99)
    codes, b = R.quantize(x)
    assert np.all(b == 127)
    v = R.values(codes, b)
    nearest = np.abs(x[..., None] - np.concatenate([R.GRID, -R.GRID])).min(-1)
    np.testing.assert_array_equal(np.abs(x - v), nearest)
    ties = np.zeros((1, 32))
    ties[0, :10] = [4, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -2.5, 7.9]
    np.testing.assert_array_equal(R.values(*R.quantize(ties))[0, :10], [4, 0, 1, 1, 2, 2, 4, 4, -2, 6])


def test_reference_scales_and_packing():
    x = np.zeros((5, 544))
    x[0, 0], x[1, 33], x[2, 64], x[3, 100] = 1.0, 7.9, 2.0 ** -140, np.inf
    b = R.scale_bytes(x)
    assert (b[0, 0], b[1, 1], b[2, 2], b[3, 3], b[4, 0]) == (125, 127, 0, 255, 0)
    codes, b = R.quantize(x)
    q, s = R.pack(codes, b)
    assert q.shape == (5, 272) and s.shape == (5, 32) and cat.cat_mx_scale_pitch(544) == 32
    assert not s[:, 17:].any()
    again = R.unpack(q, s)
    np.testing.assert_array_equal(again[0], codes)
    np.testing.assert_array_equal(again[1], b)


def test_scale_pitch(lib):
    for d in (32, 480, 512, 544, 4096, 14336, 262144):
        assert lib.cat_mx_scale_pitch(d) == cat.cat_mx_scale_pitch(d) == R.pitch(d) and R.pitch(d) % 16 == 0
        assert R.pitch(d) >= d // 32
    for d in (0, -32, 48, 262176):
        assert lib.cat_mx_scale_pitch(d) == 0


def test_refusals(lib):
    """Invalid calls are refused on the host, before anything touches CUDA."""
    # (x, dtype, n, d, rows, m, xq, xs, stream)
    q = lib.cat_mx_quantize
    assert q(P, 2, 4, 64, None, 4, P, P, None) == 1                 # dtype
    assert q(P, 0, 4, 48, None, 4, P, P, None) == 2                 # d % 32
    assert q(P, 0, 4, 0, None, 4, P, P, None) == 2
    assert q(P, 0, 4, 262176, None, 4, P, P, None) == 2             # too long a row
    assert q(P, 0, -1, 64, None, -1, P, P, None) == 2
    assert q(P, 0, 4, 64, None, 5, P, P, None) == 2                 # m without rows
    assert q(P, 0, 4, 64, P, -1, P, P, None) == 2
    assert q(P, 0, 1 << 31, 64, None, 1 << 31, P, P, None) == 2
    assert q(None, 0, 4, 64, None, 4, P, P, None) == 1
    assert q(P, 0, 4, 64, None, 4, None, P, None) == 1
    assert q(P, 0, 4, 64, None, 4, P, None, None) == 1
    for bad in ((BAD, None, P, P), (P, BAD, P, P), (P, None, BAD, P), (P, None, P, BAD)):
        assert q(bad[0], 0, 4, 64, bad[1], 4, bad[2], bad[3], None) == 3
    assert q(None, 0, 0, 64, None, 0, None, None, None) == 0        # nothing to do
    # (xq, xs, n, d, out_dtype, out, stream)
    dq = lib.cat_mx_dequantize
    assert dq(P, P, 4, 64, 5, P, None) == 1
    assert dq(P, P, 4, 40, 0, P, None) == 2
    assert dq(P, None, 4, 64, 0, P, None) == 1
    assert dq(P, P, 4, 64, 0, BAD, None) == 3
    assert dq(None, None, 0, 64, 0, None, None) == 0
    # (gu, dtype, n, d, xq, xs, stream)
    g = lib.cat_mx_swiglu_quantize
    assert g(P, 3, 4, 64, P, P, None) == 1
    assert g(P, 1, 4, 63, P, P, None) == 2
    assert g(None, 1, 4, 64, P, P, None) == 1
    assert g(P, 1, 4, 64, P, BAD, None) == 3
    assert g(None, 1, 0, 64, None, None, None) == 0
    # (x, residual, dtype, weight, weight_dtype, n, d, eps, h, xq, xs, stream)
    r = lib.cat_mx_rmsnorm_quantize
    assert r(P, P, 2, P, 0, 4, 64, 0.1, P, P, P, None) == 1
    assert r(P, P, 0, P, 2, 4, 64, 0.1, P, P, P, None) == 1
    for eps in (-1e-6, NAN, INF):
        assert r(P, P, 0, P, 0, 4, 64, eps, P, P, P, None) == 1
    assert r(P, P, 0, P, 0, 4, 16, 0.1, P, P, P, None) == 2
    assert r(P, P, 0, None, 0, 4, 64, 0.1, P, P, P, None) == 1
    assert r(P, BAD, 0, P, 0, 4, 64, 0.1, P, P, P, None) == 3
    assert r(P, P, 0, P, 0, 4, 64, 0.1, BAD, P, P, None) == 3
    assert r(None, None, 0, None, 0, 0, 64, 0.1, None, None, None, None) == 0
    # (xq, xs, Wq, ws, n, d, d_out, out_dtype, y, stream)
    f = lib.cat_mx_linear
    assert f(P, P, P, P, 4, 64, 8, 2, P, None) == 1
    assert f(P, P, P, P, 4, 72, 8, 0, P, None) == 2
    assert f(P, P, P, P, 4, 64, 0, 0, P, None) == 2
    assert f(P, P, P, P, 4, 64, 1 << 31, 0, P, None) == 2
    assert f(P, P, P, P, 4, 64, 8, 0, None, None) == 1
    assert f(P, P, BAD, P, 4, 64, 8, 0, P, None) == 3
    assert f(None, None, None, None, 0, 64, 8, 0, None, None) == 0
    # (xq, xs, Wq, ws, offsets, experts, m, d, d_out, out_dtype, y, stream)
    e = lib.cat_mx_linear_grouped
    assert e(P, P, P, P, P, 2, 4, 64, 8, 7, P, None) == 1
    for experts in (0, -1, 1025):
        assert e(P, P, P, P, P, experts, 4, 64, 8, 0, P, None) == 2
    assert e(P, P, P, P, P, 1024, 4, 64, 1 << 22, 0, P, None) == 2  # experts x d_out
    assert e(P, P, P, P, None, 2, 4, 64, 8, 0, P, None) == 1
    assert e(P, P, P, P, BAD, 2, 4, 64, 8, 0, P, None) == 3
    assert e(P, P, P, P, P, 2, -4, 64, 8, 0, P, None) == 2
    assert e(None, None, None, None, None, 2, 0, 64, 8, 0, None, None) == 0
    f(P, P, P, P, 4, 72, 8, 0, P, None)
    assert b"multiple of 32" in lib.cat_last_error()


def test_compiled_calls_leave_other_arguments_to_the_binding(lib):
    """Tensors that are not on a GPU (or none at all) are not taken: None, and nothing has touched CUDA."""
    import torch
    calls = cat._calls()
    x, u = torch.randn(4, 64), torch.zeros(4, 32, dtype=torch.uint8)
    assert calls.quantize(x, None) is None and calls.quantize(3, None) is None and calls.swiglu_quantize(x) is None
    assert calls.rmsnorm_quantize(x, x[0], 1e-5, None) is None and calls.dequantize(u, u, None) is None
    assert calls.linear(u, u, u, u, None) is None and calls.linear_grouped(u, u, u, u, u, torch.float32) is None
    with pytest.raises(TypeError):
        calls.quantize(x)
    with pytest.raises(ValueError):
        cat.cat_mx_quantize(x)


A = 0x10 << 40          # an address that holds nothing


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeRuntime(tmp_path_factory.mktemp("fake_mx"))


def form(launch):
    """pairs or single CTAs, CTAs a cluster."""
    cg = 2 if "mx_gemm_kernel<2" in launch.kernel else 1
    return (cg, launch.cluster, launch.grid)


@pytest.mark.parametrize("n,d,d_out,cg,cluster,grid", [
    (1, 4096, 6144, 1, 2, 96), (1, 4096, 4096, 1, 4, 128), (27, 14336, 4096, 1, 4, 128), (16, 4096, 14336, 1, 1, 112),
    (1, 8192, 28672, 1, 1, 152), (128, 14336, 4096, 1, 4, 128), (200, 4096, 14336, 2, 2, 112), (201, 4096, 6144, 1, 1, 144),
    (512, 4096, 4096, 1, 1, 128), (2048, 4096, 6144, 2, 2, 152), (8192, 8192, 28672, 2, 2, 152), (1, 256, 256, 1, 1, 2),
])
def test_products_take_the_form_of_least_time(fake, n, d, d_out, cg, cluster, grid):
    """The forms that were measured fastest, on 152 SMs."""
    launch, = fake.call("cat_mx_linear", A, A, A, A, n, d, d_out, 1, A, None)
    assert form(launch) == (cg, cluster, grid)
    # a cluster leaves no room on its SMs for another kernel's CTA with tensor memory of its own
    assert launch.smem >= (215 if cluster > 1 else 120) * 1024


def mx_calls(fake):
    for dtype in (0, 1):
        for n, d in ((1, 32), (3, 4096), (5000, 8192), (2, 262144)):
            yield "cat_mx_quantize", A, dtype, n, d, None, n, A, A, None
            yield "cat_mx_quantize", A, dtype, n, d, A, 2 * n, A, A, None
            yield "cat_mx_swiglu_quantize", A, dtype, n, d, A, A, None
            yield "cat_mx_dequantize", A, A, n, d, dtype, A, None
            for weight in (0, 1):
                yield "cat_mx_rmsnorm_quantize", A, A, dtype, A, weight, n, d, 1e-5, A, A, A, None
        for n, d, d_out in ((1, 32, 1), (1, 4096, 4096), (1, 4096, 1000), (40, 4096, 6144), (300, 1120, 4097), (5000, 14336, 8192)):
            yield "cat_mx_linear", A, A, A, A, n, d, d_out, dtype, A, None
            for experts in (1, 7, 1024):
                yield "cat_mx_linear_grouped", A, A, A, A, A, experts, n, d, d_out, dtype, A, None


def test_every_launch_is_allowed_on_every_device(fake):
    first, second = [], []
    for found, device in ((first, 2), (second, 6)):
        fake.device(device)
        for name, *args in mx_calls(fake):
            launches = fake.call(name, *args)
            assert len(launches) == 1, (name, args)                 # one launch a call, without scratch or memsets
            found += launches
    fake.device(0)
    assert [x._replace(device=0) for x in first] == [x._replace(device=0) for x in second]
    assert {x.device for x in second} == {6}


@pytest.mark.parametrize("n,d_out,groups,rows", [(1, 6144, None, [128, 8, 128, 8]), (201, 6144, None, [128, 72, 128, 72]),
                                                 (8192, 28672, None, [128, 128, 128, 256]), (16, 14336, 8, [128, 8, 128, 8]),
                                                 (4096, 14336, 8, [128, 64, 128, 64])])
def test_products_load_the_token_rows_there_are(fake, n, d_out, groups, rows):
    """Boxes: the weights' codes, the tokens', and the same of the scales."""
    if groups:
        fake.call("cat_mx_linear_grouped", A, A, A, A, A, groups, n, 4096, d_out, 1, A, None)
    else:
        fake.call("cat_mx_linear", A, A, A, A, n, 4096 if n < 8192 else 8192, d_out, 1, A, None)
    assert fake.box_rows() == rows
