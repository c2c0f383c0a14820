"""The products' exact comparison itself: an output that lacks one step of K, one part of a split or one block is refused."""
import numpy as np
import pytest
import torch

import mx_products as M
import mx_reference as R


@pytest.mark.parametrize("n,d,d_out", [(40, 131072, 64), (16, 65536, 64), (27, 14336, 64), (3, 512, 40)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_lost_is_refused(n, d, d_out, dtype):
    rng = np.random.default_rng(d)
    xq, xs = M.operand(rng, n, d, M.binades(d))
    wq, ws = M.operand(rng, d_out, d, M.binades(d))
    want = M.expected(xq, xs, wq, ws)
    M.check(want.float().to(dtype), want)
    x, w = M.values(xq, xs, "cpu")[0], M.values(wq, ws, "cpu")[0]
    for lost in (slice(d - d // 8, d), slice(256, 512), slice(d - 32, d)):      # a split's part, a step of K, a block
        with pytest.raises(AssertionError, match="outputs differ"):
            M.check((want - x[:, lost] @ w[:, lost].T).float().to(dtype), want)
    one = want.clone()
    one[n - 1, d_out - 1] += 2.0 if dtype is torch.bfloat16 and d < 1024 else float(one.abs().max()) / 16
    with pytest.raises(AssertionError, match="1 of"):
        M.check(one.float().to(dtype), want)


def test_sums_have_to_be_exact():
    rng = np.random.default_rng(0)
    xq, xs = M.operand(rng, 4, 4096, 9)
    with pytest.raises(AssertionError, match="other operands"):
        M.expected(xq, xs, xq, xs)


def test_float32_sums_of_the_operands_are_exact_in_any_order():
    rng = np.random.default_rng(1)
    for d in (32, 4096, 14336, 65536, 131072):
        xq, xs = M.operand(rng, 8, d, M.binades(d))
        wq, ws = M.operand(rng, 8, d, M.binades(d))
        want = M.expected(xq, xs, wq, ws)
        x, w = (R.values(*R.unpack(q.numpy(), s.numpy())).astype(np.float32) for q, s in ((xq, xs), (wq, ws)))
        p = x[:, None] * w[None]
        for order in (np.arange(d), rng.permutation(d)):
            assert np.array_equal(np.cumsum(p[..., order], -1, dtype=np.float32)[..., -1], want.numpy())
