"""A decoder block's mixture-of-experts half in microscaled 4-bit arithmetic (MXFP4 weights and activations).

    h = x + residual;  v = RMSnorm(h);  experts of the top router logits;  y = h + sum_e p_e down_e(SwiGLU(gate_up_e(v)))

Every product, the router's too, runs on 4-bit operands: the norm and SwiGLU write the 4-bit form of their output straight away, tokens are
dispatched as 4-bit rows, and the experts' products take ragged groups from offsets on the device, so nothing waits for
the host between the norm and the result.

    python examples/mx_experts.py [--tokens 256] [--width 1024] [--hidden 2048] [--experts 8] [--top 2]

prints the signal-to-quantization-noise ratio of the experts' output against the same experts in float32 on the same routing:
what the 4-bit router chooses otherwise than a float32 one is not part of it.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_04359_gb300 as cat  # noqa: E402


class Experts:
    """Weights of the block: gain [width], router [experts, width], gate_up [experts, 2 hidden, width] (rows of the gate,
    then of u), down [experts, width, hidden], kept in the 4-bit form."""

    def __init__(self, gain, router, gate_up, down, top, eps=1e-5):
        self.gain, self.top, self.eps = gain, top, eps
        self.router = cat.cat_mx_quantize(router)
        self.gate_up = self._prepared(gate_up)
        self.down = self._prepared(down)

    @staticmethod
    def _prepared(w):
        codes, scales = cat.cat_mx_quantize(w.reshape(-1, w.shape[-1]))
        return codes.view(*w.shape[:-1], -1), scales.view(*w.shape[:-1], -1)

    def route(self, logits):
        """(rows int32 [n top]: the token of each dispatched row, in the experts' order; offsets int32 [experts + 1];
        shares float32 [n top] of the rows)."""
        shares, chosen = torch.topk(torch.softmax(logits, -1), self.top, dim=-1)
        order = torch.argsort(chosen.reshape(-1), stable=True)
        sizes = torch.zeros(logits.shape[-1] + 1, dtype=torch.int32, device=logits.device)
        sizes.scatter_add_(0, chosen.reshape(-1) + 1, torch.ones_like(order, dtype=torch.int32))
        return (order // self.top).int(), sizes.cumsum(0, dtype=torch.int32), shares.reshape(-1)[order]

    def __call__(self, x, residual):
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(x, self.gain, self.eps, residual=residual)
        rows, offsets, shares = self.route(cat.cat_mx_linear(xq, xs, *self.router))
        gu = cat.cat_mx_linear_grouped(xq[rows], xs[rows], *self.gate_up, offsets, out_dtype=torch.bfloat16)
        out = cat.cat_mx_linear_grouped(*cat.cat_mx_swiglu_quantize(gu), *self.down, offsets)
        # a token's rows, in the order of its experts: summed in that order, the same each time
        mine = torch.argsort(rows, stable=True).view(-1, self.top)
        return h.float() + (out * shares[:, None])[mine].sum(1), (rows, offsets, shares)


def reference(x, residual, gain, gate_up, down, routing, eps=1e-5):
    """The same block in float32 with unquantized weights, on the routing that the 4-bit block took."""
    rows, offsets, shares = routing
    h = x.float() + residual.float()
    v = (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * gain.float())[rows]
    edges = offsets.tolist()
    y = h.to(x.dtype).float()
    for e, (lo, hi) in enumerate(zip(edges, edges[1:])):
        gate, u = (v[lo:hi] @ gate_up[e].float().T).chunk(2, -1)
        out = (torch.nn.functional.silu(gate) * u) @ down[e].float().T
        y.index_add_(0, rows[lo:hi], out * shares[lo:hi, None])
    return y


def run(tokens, width, hidden, experts, top, seed=0, device="cuda"):
    """(4-bit output, float32 output, the block's part of each without h, SQNR in dB of that part)."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def randn(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g, device=device)).to(torch.bfloat16)
    gain, router = 1 + randn(width, scale=0.1), randn(experts, width, scale=width ** -0.5)
    gate_up, down = randn(experts, 2 * hidden, width, scale=width ** -0.5), randn(experts, width, hidden, scale=hidden ** -0.5)
    x, residual = randn(tokens, width), randn(tokens, width)
    y, routing = Experts(gain, router, gate_up, down, top)(x, residual)
    ref = reference(x, residual, gain, gate_up, down, routing)
    h = (x.float() + residual.float()).to(x.dtype).float()
    parts = (y - h).contiguous(), (ref - h).contiguous()
    return y, ref, parts, float(cat.cat_sqnr(parts[1], parts[0])[2])


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 256), ("width", 1024), ("hidden", 2048), ("experts", 8), ("top", 2)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args()
    y, _, _, db = run(a.tokens, a.width, a.hidden, a.experts, a.top)
    status, word = cat.cat_device_status()
    print(f"{a.tokens} tokens, {a.width} wide, {a.experts} experts of {a.hidden}, {a.top} a token: experts' output at "
          f"{db:.2f} dB SQNR against float32, status {status}")
    return 0 if status == 0 and bool(torch.isfinite(y).all()) else 1


if __name__ == "__main__":
    sys.exit(main())
