"""Calls that are the first CUDA work of their thread: the device's context is not current there yet."""
import threading

import numpy as np
import pytest
import torch

import dp_planes

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")
DEV = "cuda"


def codes(rows, d):
    rng = np.random.default_rng(rows + d)
    return (torch.from_numpy(rng.integers(0, 256, (rows, d // 2), dtype=np.uint8)).to(DEV),
            torch.rand(rows, device=DEV) + 0.5)


def empty(dtype, *shape):
    return torch.empty(shape, dtype=dtype, device=DEV)


def covariance():
    x, out = torch.randn(512, 1024, device=DEV).bfloat16(), empty(torch.float64, 8, 128, 128)
    return lambda: cat.cat_calib_cov(x, 128, out=out)


def transform(n):
    def make():
        x, T = torch.randn(n, 1024, device=DEV).bfloat16(), torch.randn(8, 128, 128, device=DEV)
        q, s = empty(torch.uint8, n, 512), empty(torch.float32, n)
        return lambda: cat.cat_transform_quantize_act(x, T, 128, xq=q, x_scale=s)
    return make


def integer(n, as_bytes):
    def make():
        (xq, sx), (wq, sw) = codes(n, 1024), codes(640, 1024)
        if as_bytes:
            xq, wq = cat.cat_codes_to_e4m3(xq), cat.cat_codes_to_e4m3(wq)
        y = empty(torch.float32, n, 640)
        return lambda: (cat.cat_w4a4_linear_e8 if as_bytes else cat.cat_w4a4_linear)(xq, sx, wq, sw, y=y)
    return make


def planes():
    rng = np.random.default_rng(3)
    xp, wp = (torch.from_numpy(dp_planes.encode(rng.integers(-7, 8, (r, 1024)), 4, False)).to(DEV) for r in (200, 640))
    sx, sw, y = torch.rand(200, device=DEV), torch.rand(640, device=DEV), empty(torch.float32, 200, 640)
    return lambda: cat.cat_linear_dp(xp, 4, sx, wp, 4, sw, y=y)


def microscaled(n, groups):
    def make():
        xq, xs = cat.cat_mx_quantize(torch.randn(n, 1024, device=DEV))
        wq, ws = cat.cat_mx_quantize(torch.randn(2 * 320, 1024, device=DEV))
        if not groups:
            y = empty(torch.float32, n, 640)
            return lambda: cat.cat_mx_linear(xq, xs, wq, ws, y=y)
        ends = torch.tensor([0, n // 3, n], dtype=torch.int32, device=DEV)
        wq, ws, y = wq.view(2, 320, -1), ws.view(2, 320, -1), empty(torch.float32, n, 320)
        return lambda: cat.cat_mx_linear_grouped(xq, xs, wq, ws, ends, y=y)
    return make


CALLS = {"covariance": covariance, "transform 16": transform(16), "transform 400": transform(400), "integer 8": integer(8, False),
         "integer 300": integer(300, False), "bytes 300": integer(300, True), "planes": planes, "microscaled 1": microscaled(1, False),
         "microscaled 1500": microscaled(1500, False), "experts": microscaled(40, True)}


@pytest.mark.parametrize("name", CALLS)
def test_first_cuda_work_of_a_thread(name):
    call = CALLS[name]()
    flat = lambda r: r if isinstance(r, tuple) else (r,)   # noqa: E731
    out = flat(call())
    want = [t.clone() for t in out]
    for t in out:
        t.zero_()
    torch.cuda.synchronize()
    wrong = []

    def work():
        try:
            call()
        except Exception as e:
            wrong.append(e)
    thread = threading.Thread(target=work)
    thread.start()
    thread.join()
    assert not wrong, wrong
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert cat.cat_device_status()[0] == 0
