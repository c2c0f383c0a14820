"""The binding refuses tensors of a device that is not the current one.

The library launches on the current device: with another device's tensors a kernel would get pointers that are not its
own's.  Shown without a GPU: tensors that say they are on cuda:1 (over host memory), in a process whose CUDA runtime
says that cuda:0 is current (two functions in front of the runtime's)."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2603_04359_gb300 as cat
from fake_runtime import ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import ctypes, torch
import paper_2603_04359_gb300 as cat

def on(device, dtype, *shape):
    n = empty(shape, dtype=dtype).nbytes
    kept.append((ctypes.c_char * max(n, 16))())
    s = torch._C._construct_storage_from_data_pointer(ctypes.addressof(kept[-1]), torch.device("cuda", device), n)
    stride = [1] * len(shape)
    for i in range(len(shape) - 2, -1, -1):
        stride[i] = stride[i + 1] * shape[i + 1]
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        dict(size=shape, stride=tuple(stride), dtype=dtype, storage_offset=0), s)

torch._C._cuda_getDevice = lambda: 0          # (torch's own wants a driver first)
empty = torch.empty
torch.empty = lambda shape, dtype, device: on(device.index, dtype, *shape)
kept = []
f, u, i = torch.float32, torch.uint8, torch.int32
x, x2, w = on(1, f, 4, 64), on(1, f, 4, 128), on(1, f, 64)
q, s, wq, ws, o = on(1, u, 4, 32), on(1, u, 4, 16), on(1, u, 2, 8, 32), on(1, u, 2, 8, 16), on(1, i, 3)
w1, s1 = on(1, u, 8, 32), on(1, u, 8, 16)
calls = {
    "quantize": lambda: cat.cat_mx_quantize(x),
    "quantize to buffers": lambda: cat.cat_mx_quantize(x, xq=q, xs=s),
    "gather": lambda: cat.cat_mx_quantize(x, rows=o, xq=on(1, u, 3, 32), xs=on(1, u, 3, 16)),
    "swiglu": lambda: cat.cat_mx_swiglu_quantize(x2),
    "swiglu to buffers": lambda: cat.cat_mx_swiglu_quantize(x2, xq=q, xs=s),
    "norm": lambda: cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=x),
    "norm to buffers": lambda: cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=x, h=x, xq=q, xs=s),
    "dequantize": lambda: cat.cat_mx_dequantize(q, s),
    "dequantize to a buffer": lambda: cat.cat_mx_dequantize(q, s, out=x),
    "linear": lambda: cat.cat_mx_linear(q, s, w1, s1),
    "linear to a buffer": lambda: cat.cat_mx_linear(q, s, w1, s1, y=on(1, f, 4, 8)),
    "grouped": lambda: cat.cat_mx_linear_grouped(q, s, wq, ws, o),
    "grouped to a buffer": lambda: cat.cat_mx_linear_grouped(q, s, wq, ws, o, y=on(1, f, 4, 8)),
    "covariance": lambda: cat.cat_calib_cov(x, 32, out=on(1, torch.float64, 2, 32, 32)),
}
for name, call in calls.items():
    try:
        call()
    except BaseException as e:
        print(name, "|", type(e).__name__, "|", e)
    else:
        print(name, "| went through |")
native = cat._calls()
for r in (native.quantize(x, None), native.swiglu_quantize(x2), native.rmsnorm_quantize(x, w, 1e-5, x), native.dequantize(q, s, f),
          native.linear(q, s, w1, s1, f), native.linear_grouped(q, s, wq, ws, o, f)):
    print("compiled |", "left to the binding" if r is None else r, "|")
"""


@pytest.fixture(scope="module")
def outcome(tmp_path_factory):
    ensure_built()
    folder = tmp_path_factory.mktemp("device")
    lib = os.path.join(str(folder), "current.so")
    source = os.path.join(str(folder), "current.c")
    with open(source, "w") as f:
        f.write("int cudaGetDevice(int* d) { *d = 0; return 0; }\nint cudaGetDeviceCount(int* n) { *n = 0; return 0; }\n")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", lib, source], check=True)
    p = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, capture_output=True, text=True,
                       env=dict(os.environ, LD_PRELOAD=lib, CUDA_VISIBLE_DEVICES=""))
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]
    return [[part.strip() for part in line.split("|")] for line in p.stdout.splitlines()]


def test_every_call_says_which_device_is_current(outcome):
    calls = [r for r in outcome if r[0] != "compiled"]
    assert len(calls) == 14
    for name, kind, message in calls:
        assert kind == "ValueError" and "cuda:1" in message and "the current device is cuda:0" in message, (name, kind, message)


def test_compiled_calls_leave_them_to_the_binding(outcome):
    compiled = [r for r in outcome if r[0] == "compiled"]
    assert len(compiled) == 6 and all(r[1] == "left to the binding" for r in compiled), compiled


def test_stream_of_the_current_device(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3)
    monkeypatch.setattr(cat, "_raw_stream", lambda index: 100 + index)
    assert cat._stream(torch.device("cuda", 3)) == 103
    with pytest.raises(ValueError, match="cuda:0.*current device is cuda:3"):
        cat._stream(torch.device("cuda", 0))
