"""The microscaled row operators on tensors that lie on 16 bytes but not on 32, where rows are moved 16 bytes at a time:
the same bytes as on a fresh allocation, and nothing written around them."""
import numpy as np
import pytest
import torch

from test_gpu_mx import TYPES, cat, dev, tokens

pytestmark = pytest.mark.gpu
DEV = "cuda"
GUARD = 0x5C


class Shifted:
    """Room for a tensor that begins 16 bytes into a buffer; guard bytes on both sides."""

    def __init__(self, dtype, *shape):
        self.nbytes = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.buffer = torch.full((self.nbytes + 512,), GUARD, dtype=torch.uint8, device=DEV)
        self.at = 240
        self.t = self.buffer[self.at:self.at + self.nbytes].view(dtype).view(shape)
        assert self.t.data_ptr() % 32 == 16

    def whole(self):
        return bool((self.buffer[:self.at] == GUARD).all()) and bool((self.buffer[self.at + self.nbytes:] == GUARD).all())


def shifted(t):
    s = Shifted(t.dtype, *t.shape)
    s.t.copy_(t)
    return s


def form(n, d):
    return Shifted(torch.uint8, n, d // 2), Shifted(torch.uint8, n, cat.cat_mx_scale_pitch(d))


def same(got, want):
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1, 32), (7, 480), (33, 544), (300, 4096)])
def test_quantize_gather_swiglu_dequantize(n, d, dtype):
    rng = np.random.default_rng(n + d)
    x = dev(tokens(rng, n, d), TYPES[dtype])
    rows = dev(rng.integers(-1, n, 2 * n + 1).astype(np.int32))
    gu = dev(rng.standard_normal((n, 2 * d)), TYPES[dtype])
    for call, given, m in ((cat.cat_mx_quantize, x, n), (lambda t, **k: cat.cat_mx_quantize(t, rows=rows, **k), x, 2 * n + 1),
                           (cat.cat_mx_swiglu_quantize, gu, n)):
        want = call(given)
        source, (q, s) = shifted(given), form(m, d)
        same(call(source.t, xq=q.t, xs=s.t), want)                  # the input and what is written
        same(call(given, xq=q.t, xs=s.t), want)
        same(call(source.t), want)
        assert source.whole() and q.whole() and s.whole() and torch.equal(source.t, given)
    q, s = cat.cat_mx_quantize(x)
    for out in TYPES.values():
        want, to = cat.cat_mx_dequantize(q, s, out_dtype=out), Shifted(out, n, d)
        assert torch.equal(cat.cat_mx_dequantize(q, s, out=to.t), want) and to.whole()
        to.t.fill_(float("nan"))
        assert torch.equal(cat.cat_mx_dequantize(shifted(q).t, shifted(s).t, out=to.t), want) and to.whole()
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("dtype,weight", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,d", [(5, 96), (4, 512), (700, 4096), (3, 9024), (3, 14336), (2, 40000)])
def test_norm(n, d, dtype, weight):
    """A warp a row, a CTA a row with one and with two halves a thread, two readings; one tensor shifted at a time."""
    rng = np.random.default_rng(n + d)
    x, r = dev(tokens(rng, n, d), TYPES[dtype]), dev(rng.standard_normal((n, d)), TYPES[dtype])
    w = dev(1 + 0.2 * rng.standard_normal(d), TYPES[weight])
    want = cat.cat_mx_rmsnorm_quantize(x, w, 1e-5, residual=r)
    plain = cat.cat_mx_rmsnorm_quantize(x, w, 1e-5)
    for which in ("x", "residual", "weight", "h", "all"):
        mine = lambda name, t: shifted(t).t if which in (name, "all") else t  # noqa: E731
        h, (q, s) = Shifted(x.dtype, n, d), form(n, d)
        to = dict(h=h.t) if which in ("h", "all") else {}
        if which == "all":
            to.update(xq=q.t, xs=s.t)
        same(cat.cat_mx_rmsnorm_quantize(mine("x", x), mine("weight", w), 1e-5, residual=mine("residual", r), **to), want)
        same(cat.cat_mx_rmsnorm_quantize(mine("x", x), mine("weight", w), 1e-5)[:2], plain[:2])
        assert h.whole() and q.whole() and s.whole()
    for name in ("x", "residual"):                                  # the sum over one of them
        a, b = shifted(x), shifted(r)
        over = a if name == "x" else b
        same(cat.cat_mx_rmsnorm_quantize(a.t, w, 1e-5, residual=b.t, h=over.t), want)
        assert a.whole() and b.whole()
    assert cat.cat_device_status()[0] == 0


@pytest.mark.parametrize("n,d,d_out", [(3, 64, 40), (300, 1056, 512)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_products(n, d, d_out, out):
    """Every operand and y, one at a time (rows that a copy starts 16 bytes into a line)."""
    rng = np.random.default_rng(d)
    given = [*cat.cat_mx_quantize(dev(rng.standard_normal((n, d)), torch.float32)),
             *cat.cat_mx_quantize(dev(rng.standard_normal((d_out, d)), torch.float32))]
    want = cat.cat_mx_linear(*given, out_dtype=TYPES[out])
    for i in range(5):
        y = Shifted(TYPES[out], n, d_out)
        a = [shifted(t).t if i == j else t for j, t in enumerate(given)]
        got = cat.cat_mx_linear(*a, y=y.t) if i == 4 else cat.cat_mx_linear(*a, out_dtype=TYPES[out])
        assert torch.equal(got, want) and y.whole()
    assert cat.cat_device_status()[0] == 0
