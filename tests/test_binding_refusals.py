"""The two copies of the microscaled calls' checks agree: what the compiled calls do not take (they return None) the Python
functions refuse with ValueError or TypeError, and the valid calls pass both (they fail at the first allocation or launch
on a machine without a GPU)."""
import pytest

import host_tensors

SCRIPT = """
torch.empty = lambda shape, dtype, device: on(device.index, dtype, *shape)
native = cat._calls()
x, xb, w, wb = on(0, f, 4, 64), on(0, b, 4, 64), on(0, f, 64), on(0, b, 64)
q, s, r = on(0, u, 4, 32), on(0, u, 4, 16), on(0, i, 6)
wq, ws = on(0, u, 8, 32), on(0, u, 8, 16)
eq, es, o = on(0, u, 2, 8, 32), on(0, u, 2, 8, 16), on(0, i, 3)
part = on(0, f, 4, 64, stride=(128, 1))                # not contiguous
cpu = torch.zeros(4, 64)
qc, sc = torch.zeros(4, 32, dtype=u), torch.zeros(4, 16, dtype=u)

valid = {
    "quantize": [(x, None), (xb, None), (x, r), (on(0, f, 0, 64), r)],
    "swiglu_quantize": [(x,), (xb,)],
    "rmsnorm_quantize": [(x, w, 1e-5, None), (xb, w, 1e-5, xb), (x, wb, 0.0, x)],
    "dequantize": [(q, s, None), (q, s, b), (q, s, f)],
    "linear": [(q, s, wq, ws, None), (q, s, wq, ws, b)],
    "linear_grouped": [(q, s, eq, es, o, None), (q, s, eq, es, o, b)],
}
others = {
    "quantize": [(on(0, h, 4, 64), None), (on(0, torch.float64, 4, 64), None), (part, None), (cpu, None), (on(1, f, 4, 64), None),
                 (x, on(0, l, 6)), (x, on(0, f, 6)), (x, on(1, i, 6)), (x, on(0, i, 3, stride=(2,))), (x, on(0, i, 2, 3)), (x, torch.zeros(6, dtype=i)),
                 (x, [0, 1])],
    "swiglu_quantize": [(on(0, h, 4, 64),), (part,), (cpu,), (on(0, f, 4, 65),), (on(1, f, 4, 64),)],
    "rmsnorm_quantize": [(on(0, h, 4, 64), w, 1e-5, None), (x, on(0, h, 64), 1e-5, None), (x, on(0, f, 32), 1e-5, None),
                         (x, on(0, f, 1, 64), 1e-5, None), (x, on(1, f, 64), 1e-5, None), (x, torch.ones(64), 1e-5, None),
                         (x, w, 1e-5, xb), (x, w, 1e-5, on(0, f, 2, 64)), (x, w, 1e-5, on(1, f, 4, 64)), (x, w, 1e-5, part),
                         (part, w, 1e-5, None), (cpu, w, 1e-5, None), (x, w, 1e-5, cpu), (x, w, "1e-5", None)],
    "dequantize": [(qc, sc, None), (q, sc, None), (q, on(0, u, 4, 32), None), (q, on(0, u, 3, 16), None), (on(0, f, 4, 32), s, None),
                   (q, on(0, i, 4, 16), None), (q, s, h), (on(0, u, 4, 32, stride=(64, 1)), s, None), (q, on(1, u, 4, 16), None),
                   (on(1, u, 4, 32), on(1, u, 4, 16), None)],
    "linear": [(q, s, on(0, u, 8, 16), ws, None), (q, s, wq, on(0, u, 8, 32), None), (q, s, wq, on(0, u, 7, 16), None),
               (q, s, on(1, u, 8, 32), ws, None), (q, s, wq, on(1, u, 8, 16), None), (q, s, wq, ws, h), (q, s, on(0, f, 8, 32), ws, None),
               (q, s, on(0, u, 8, 32, stride=(1, 8)), ws, None), (qc, sc, wq, ws, None), (q, s, qc, sc, None), (q, s, on(0, u, 8, 2, 16), ws, None)],
    "linear_grouped": [(q, s, wq, ws, o, None), (q, s, eq, es, on(0, i, 2), None), (q, s, eq, es, on(0, l, 3), None),
                       (q, s, eq, es, on(1, i, 3), None), (q, s, eq, es, torch.zeros(3, dtype=i), None), (q, s, eq, es, on(0, i, 3, stride=(2,)), None),
                       (q, s, eq, on(0, u, 2, 7, 16), o, None), (q, s, eq, on(0, u, 1, 8, 16), o, None), (q, s, on(0, u, 2, 8, 16), es, o, None),
                       (q, s, eq, es, o, h), (q, s, eq, es, [0, 2, 4], None), (q, on(0, u, 4, 32), eq, es, o, None)],
}
python = {
    "quantize": cat.cat_mx_quantize, "swiglu_quantize": cat.cat_mx_swiglu_quantize, "dequantize": cat.cat_mx_dequantize,
    "rmsnorm_quantize": cat.cat_mx_rmsnorm_quantize, "linear": cat.cat_mx_linear, "linear_grouped": cat.cat_mx_linear_grouped}
for kind, sets in (("valid", valid), ("other", others)):
    for name, calls in sets.items():
        for k, a in enumerate(calls):
            print(kind, "|", name, k, "| compiled |", outcome(lambda: getattr(native, name)(*a)))
            print(kind, "|", name, k, "| python |", outcome(lambda: python[name](*a)))
"""


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    return host_tensors.run(SCRIPT, tmp_path_factory.mktemp("refusals"))


def test_valid_calls_pass_the_checks(outcomes):
    rows = [r for r in outcomes if r[0] == "valid"]
    assert len(rows) == 32
    for r in rows:
        assert r[3] == "AcceleratorError" and "driver" in r[4], r


def test_other_calls_pass_neither(outcomes):
    rows = [r for r in outcomes if r[0] == "other"]
    assert len(rows) == 128
    for r in rows:
        if r[2] == "compiled":
            assert (r[3], r[4]) == ("returned", "None") or r[3] == "TypeError", r
        else:
            assert r[3] in ("ValueError", "TypeError"), r
