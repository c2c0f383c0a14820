"""Other Python threads run while a microscaled call waits for room in the launch queue."""
import threading
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")


def calls():
    """One call of each operator, its outputs allocated by the call."""
    x = torch.randn(8, 256, device="cuda")
    w = torch.ones(256, device="cuda")
    q, s = cat.cat_mx_quantize(x)
    ends = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    wq, ws = torch.stack([q, q]), torch.stack([s, s])
    return {"quantize": lambda: cat.cat_mx_quantize(x), "swiglu": lambda: cat.cat_mx_swiglu_quantize(x),
            "norm": lambda: cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=x), "dequantize": lambda: cat.cat_mx_dequantize(q, s),
            "linear": lambda: cat.cat_mx_linear(q, s, q, s), "grouped": lambda: cat.cat_mx_linear_grouped(q, s, wq, ws, ends)}


@pytest.mark.parametrize("name", ["quantize", "swiglu", "norm", "dequantize", "linear", "grouped"])
def test_other_threads_run_while_a_call_waits_for_the_launch_queue(name):
    """A thread makes more calls than the queue holds behind a kernel of about half a second; this one looks at the clock."""
    call = calls()[name]
    call()
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)                     # (cycles)
    thread = threading.Thread(target=lambda: [call() for _ in range(3000)])
    begin = last = time.perf_counter()
    longest = 0.0
    thread.start()
    while thread.is_alive():
        time.sleep(0.001)
        now = time.perf_counter()
        longest, last = max(longest, now - last), now
    took = last - begin
    torch.cuda.synchronize()
    assert took > 0.2, "the queue never filled"
    assert longest < took / 4, f"stopped for {longest:.3f} of {took:.3f} s"
