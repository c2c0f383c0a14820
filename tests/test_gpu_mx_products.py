"""Products of microscaled operands to the bit: operands whose float32 sums are exact (mx_products.py), where a bound that
grows with d would not see a lost step of K or a lost part of a split."""
import numpy as np
import pytest
import torch

import mx_products as M
from test_gpu_mx import GROUPS, SHAPES, TYPES, cat, dev

pytestmark = pytest.mark.gpu
DEV = "cuda"


def operands(rng, n, rows, d):
    return tuple(t.to(DEV) for r in (n, rows) for t in M.operand(rng, r, d, M.binades(d)))


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,d_out", SHAPES + [(1, 8192, 28672), (1, 14336, 4096), (27, 14336, 4096), (128, 14336, 4096),
                                                (40, 131072, 1024), (512, 4096, 4096)])
def test_linear(n, d, d_out, out):
    a = operands(np.random.default_rng(n + d + d_out), n, d_out, d)
    M.check(cat.cat_mx_linear(*a, out_dtype=TYPES[out]), M.expected(*a, DEV))
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("counts,d,d_out", GROUPS + [([2, 0, 1], 14336, 1000), ([40], 65536, 256)],
                         ids=lambda v: str(sum(v)) + "in" + str(len(v)) if isinstance(v, list) else str(v))
def test_grouped_is_the_linear_of_each_group(counts, d, d_out, out):
    rng = np.random.default_rng(sum(counts) + d)
    m, experts = sum(counts) + 5, len(counts)
    edges = 2 + np.concatenate([[0], np.cumsum(counts)])
    xq, xs, wq, ws = operands(rng, m, experts * d_out, d)
    wq, ws = wq.view(experts, d_out, -1), ws.view(experts, d_out, -1)
    y = cat.cat_mx_linear_grouped(xq, xs, wq, ws, dev(edges.astype(np.int32)), out_dtype=TYPES[out])
    for e in range(experts):
        mine = slice(edges[e], edges[e + 1])
        if counts[e]:
            plain = cat.cat_mx_linear(xq[mine], xs[mine], wq[e], ws[e], out_dtype=TYPES[out])
            assert torch.equal(y[mine], plain)
            M.check(plain, M.expected(xq[mine], xs[mine], wq[e], ws[e], DEV))
    assert not y[:2].any() and not y[edges[-1]:].any()
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("n,d,d_out", [(40, 131072, 1024), (16, 65536, 8192), (1000, 65536, 4096)],
                         ids=["split", "single", "pairs"])
def test_calls_after_a_wait_that_gave_up(n, d, d_out):
    """The next calls are the one before, bit for bit, and exact."""
    a = operands(np.random.default_rng(13), n, d_out, d)
    want = M.expected(*a, DEV)
    before = cat.cat_mx_linear(*a)
    M.check(before, want)
    assert cat.cat_device_status()[0] == 0
    try:
        cat.cat_set_wait_limit_ns(1)
        cat.cat_mx_linear(*a)
        assert cat.cat_device_status()[0] == 7
    finally:
        cat.cat_set_wait_limit_ns(0)
    for _ in range(2):
        assert torch.equal(cat.cat_mx_linear(*a), before)
    assert cat.cat_device_status()[0] == 0


def test_graph_takes_the_offsets_of_each_replay():
    """Norm and experts captured once: each replay is the product of its own tokens by its own groups."""
    rng = np.random.default_rng(9)
    x, r = (torch.zeros(24, 512, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    gain = torch.ones(512, device=DEV, dtype=torch.bfloat16)
    wq, ws = (t.to(DEV) for t in M.operand(rng, 4 * 256, 512, 1))
    wq, ws = wq.view(4, 256, -1), ws.view(4, 256, -1)
    offsets = torch.zeros(5, dtype=torch.int32, device=DEV)

    def layer():
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, gain, 1e-5, residual=r)
        return xq, xs, h, cat.cat_mx_linear_grouped(xq, xs, wq, ws, offsets)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xq, xs, h, y = layer()
    for edges in ([0, 7, 7, 20, 24], [0, 0, 0, 0, 24], [2, 3, 9, 9, 20], [24, 24, 24, 24, 24]):
        x.copy_(dev(rng.standard_normal((24, 512))))
        r.copy_(dev(rng.standard_normal((24, 512))))
        offsets.copy_(dev(np.array(edges, dtype=np.int32)))
        y.fill_(float("nan"))
        graph.replay()
        assert torch.equal(h, (x.float() + r.float()).bfloat16())
        for e, (lo, hi) in enumerate(zip(edges, edges[1:])):
            if hi > lo:
                M.check(y[lo:hi], M.expected(xq[lo:hi], xs[lo:hi], wq[e], ws[e], DEV))
        assert not y[:edges[0]].any() and not y[edges[-1]:].any()
    assert cat.cat_device_status()[0] == 0
