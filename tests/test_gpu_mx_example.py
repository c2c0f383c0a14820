"""The experts' example: the same bits each time, and each token to the experts of its largest logits."""
import os
import sys

import numpy as np
import pytest
import torch

import mx_reference as R
from test_gpu_mx import cat, dev, host

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def block(tokens, width, hidden, experts, top):
    import mx_experts as E
    rng = np.random.default_rng(tokens)
    draw = lambda *s: dev(rng.standard_normal(s), torch.bfloat16)  # noqa: E731
    gain, router = 1 + 0.1 * draw(width), draw(experts, width) * width ** -0.5
    made = E.Experts(gain, router, draw(experts, 2 * hidden, width) * width ** -0.5, draw(experts, width, hidden) * hidden ** -0.5, top)
    return made, gain, draw(tokens, width), draw(tokens, width)


@pytest.mark.parametrize("tokens,width,hidden,experts,top", [(1, 256, 256, 4, 2), (1500, 512, 256, 8, 4)])
def test_same_bits_each_time(tokens, width, hidden, experts, top):
    made, _, x, r = block(tokens, width, hidden, experts, top)
    first, _ = made(x, r)
    for _ in range(10):
        assert torch.equal(made(x, r)[0], first)


@pytest.mark.parametrize("tokens,width,hidden,experts,top", [(37, 1024, 256, 8, 2), (600, 512, 256, 16, 4)])
def test_tokens_go_to_the_experts_of_their_largest_logits(tokens, width, hidden, experts, top):
    """Logits in float64 of the values that the router multiplies; a choice may differ where two logits are closer than the
    float32 sums' bound, d 2^-23 sum |v w|, on both."""
    made, gain, x, r = block(tokens, width, hidden, experts, top)
    _, (rows, offsets, shares) = made(x, r)
    xq, xs, _ = cat.cat_mx_rmsnorm_quantize(x, gain, 1e-5, residual=r)
    v = R.values(*R.unpack(xq.cpu().numpy(), xs.cpu().numpy()))
    w = R.values(*R.unpack(*(t.cpu().numpy() for t in made.router)))
    logits, slack = v @ w.T, 2 * width * 2.0 ** -23 * (np.abs(v) @ np.abs(w).T).max(1)
    rows, offsets, shares = (host(t) for t in (rows, offsets, shares))
    expert = np.repeat(np.arange(experts), np.diff(offsets))
    assert len(rows) == tokens * top and offsets[0] == 0
    p = np.exp(logits - logits.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    for t in range(tokens):
        mine = expert[rows == t]
        assert len(set(mine)) == top
        rest = np.setdiff1d(np.arange(experts), mine)
        assert logits[t, mine].min() >= logits[t, rest].max() - slack[t]
        np.testing.assert_allclose(shares[rows == t], p[t, mine], rtol=1e-4)
