"""The binding refuses tensors of a device that is not the current one.

The library launches on the current device: with another device's tensors a kernel would get pointers that are not its
own's.  Shown without a GPU by tensors that say they are on cuda:1 where cuda:0 is current (host_tensors.py)."""
import pytest
import torch

import host_tensors
import paper_2603_04359_gb300 as cat

CALLS = """
torch.empty = lambda shape, dtype, device: on(device.index, dtype, *shape)
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
    print(name, "|", outcome(call))
native = cat._calls()
for r in (native.quantize(x, None), native.swiglu_quantize(x2), native.rmsnorm_quantize(x, w, 1e-5, x), native.dequantize(q, s, f),
          native.linear(q, s, w1, s1, f), native.linear_grouped(q, s, wq, ws, o, f)):
    print("compiled |", "left to the binding" if r is None else r, "|")
"""


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    return host_tensors.run(CALLS, tmp_path_factory.mktemp("device"))


def test_every_call_says_which_device_is_current(outcomes):
    calls = [r for r in outcomes if r[0] != "compiled"]
    assert len(calls) == 14
    for name, kind, message in calls:
        assert kind == "ValueError" and "cuda:1" in message and "the current device is cuda:0" in message, (name, kind, message)


def test_compiled_calls_leave_them_to_the_binding(outcomes):
    compiled = [r for r in outcomes if r[0] == "compiled"]
    assert len(compiled) == 6 and all(r[1] == "left to the binding" for r in compiled), compiled


def test_stream_of_the_current_device(monkeypatch):
    monkeypatch.setattr(cat, "_raw_device", lambda: 3)
    monkeypatch.setattr(cat, "_raw_stream", lambda index: 100 + index)
    assert cat._stream(torch.device("cuda", 3)) == 103
    with pytest.raises(ValueError, match="cuda:0.*current device is cuda:3"):
        cat._stream(torch.device("cuda", 0))
