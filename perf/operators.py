"""What the microscaled 4-bit (MXFP4) operators are timed on, in plain torch and as the library's calls.

A case is a dict of plain values.  ``op`` names the operator that a pass goes through:

* ``quantize``: x to 4-bit values with a power-of-two scale for 32 of them, and back to the values they stand for.
* ``norm``: residual addition, root-mean-square norm and the 4-bit form of its output (returned as its values).
* ``linear``: a 4-bit linear layer, x -> y: the activations' 4-bit form, then the product with prepared weights.
* ``down``: a down projection behind SwiGLU: silu(g) u in the 4-bit form, then the product.
* ``experts``: tokens dispatched to experts: the rows' gather into the 4-bit form, then the products grouped by expert.

``own`` chooses between the plain form (32 bits, elementary operations) and the library's calls.  Weights are kept in
the 4-bit form: codes, two a byte, value 2j in the low nibble, and a row of scale bytes, padded to 16 bytes with zeros.
"""
import math

import torch

own = False
DEV = "cuda"
LARGEST = 8192 * 8192 * 28672        # multiply-adds of the largest layer listed
MOST_WEIGHTS = 8 * 14336 * 4096      # weights of the experts listed
MOST_VALUES = 28672 * 8192           # values of the largest tensor that is quantized alone


def listed():
    return [
        # a 70B gate/up projection's weights made ready, with the values that they become
        dict(name="weights_gateup", op="quantize", n=28672, d=8192, dtype="bf16", act="weights"),
        # a small float32 batch: every launch counts
        dict(name="tokens_512_f32", op="quantize", n=512, d=256, dtype="f32", act="lowrank"),
        # the norm before a projection in a ragged decode batch
        dict(name="norm_27", op="norm", n=27, d=4096, dtype="bf16", act="lowrank"),
        # the norm of a long prompt in a 70B model
        dict(name="norm_8192", op="norm", n=8192, d=8192, dtype="bf16", act="lowrank"),
        # one token through a fused QKV projection: latency
        dict(name="linear_1_qkv", op="linear", n=1, d=4096, d_out=6144, dtype="bf16", act="lowrank", out="bf16"),
        # a small decode batch through an up projection: the weights' stream
        dict(name="linear_16_up", op="linear", n=16, d=4096, d_out=14336, dtype="bf16", act="lowrank", out="f32"),
        # a short prompt chunk of odd length
        dict(name="linear_201_qkv", op="linear", n=201, d=4096, d_out=6144, dtype="bf16", act="lowrank", out="bf16"),
        # the largest: a 70B gate/up projection on a long prompt
        dict(name="linear_8192_gateup", op="linear", n=8192, d=8192, d_out=28672, dtype="bf16", act="lowrank", out="bf16"),
        # a ragged decode batch through SwiGLU and the down projection: the long contraction, few outputs
        dict(name="down_27", op="down", n=27, d=14336, d_out=4096, dtype="bf16", out="bf16"),
        # a prompt batch through SwiGLU and the down projection
        dict(name="down_4096", op="down", n=4096, d=14336, d_out=4096, dtype="bf16", out="bf16"),
        # a decode batch, each token to 2 of 8 experts
        dict(name="experts_16_of_8", op="experts", n=16, d=4096, d_out=14336, dtype="bf16", act="lowrank", out="bf16",
             experts=8, top=2, skew=0.5),
        # a prompt batch, each token to 2 of 8 experts, some of them much busier than others
        dict(name="experts_4096_of_8", op="experts", n=4096, d=4096, d_out=14336, dtype="bf16", act="lowrank", out="bf16",
             experts=8, top=2, skew=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "norm", "linear", "linear", "linear", "down", "experts", "experts"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    act = rng.choice(["lowrank", "swiglu"])
    d = 32 * max(1, _log_int(rng, 256, 14336) // 32)
    if rng.random() < 0.6:
        d = 128 * max(1, d // 128)
    if op == "quantize":
        n = min(_log_int(rng, 1, 28672), MOST_VALUES // d // (2 if dtype == "f32" else 1))
        return dict(op=op, n=n, d=d, dtype=dtype, act=rng.choice(["weights", act]))
    if op == "norm":
        n = min(_log_int(rng, 1, 8192), 8192 * 8192 // d // (2 if dtype == "f32" else 1))
        return dict(op=op, n=n, d=d, dtype=dtype, act=act)
    n, d_out = _log_int(rng, 1, 8192), _log_int(rng, 64, 28672)
    if rng.random() < 0.6:
        d_out = 32 * max(2, d_out // 32)
    # SwiGLU's product is rounded to 4 bits from values that already differ in their last bits: 16-bit outputs
    out = "bf16" if op == "down" else rng.choice(["bf16", "f32"])
    if op in ("linear", "down"):
        d_out = min(d_out, MOST_WEIGHTS // d)
        n = max(1, min(n, LARGEST // (d * d_out)))
        case = dict(op=op, n=n, d=d, d_out=d_out, dtype=dtype, out=out)
        return case if op == "down" else dict(case, act=act)
    experts = _log_int(rng, 2, 64)
    top = rng.randint(1, min(4, experts))
    d_out = max(32, min(d_out, MOST_WEIGHTS // (experts * d)))
    n = max(1, min(n, 8192 // top))
    return dict(op=op, n=n, d=d, d_out=d_out, dtype=dtype, act=act, out=out, experts=experts, top=top,
                skew=round(rng.uniform(0.0, 2.0), 2))


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _tokens(case, g, n, d):
    """Activations: 64 shared factors plus isotropic noise with 1 % of the channels a hundred times larger, SiLU(g) u,
    or the rows of a weight matrix with unequal energy."""
    act = case.get("act", "normal")
    F = _randn(g, 64, d) / 8.0
    scale = torch.ones(d, device=DEV)
    scale[torch.randperm(d, generator=g, device=DEV)[: max(1, d // 100)]] = 100.0
    out = torch.empty((n, d), dtype=_type(case["dtype"]), device=DEV)
    for i in range(0, n, 2048):
        m = min(2048, n - i)
        if act == "lowrank":
            x = (_randn(g, m, 64) @ F + math.sqrt(0.1) * _randn(g, m, d)) * scale
        elif act == "swiglu":
            a = _randn(g, m, d)
            x = a * torch.sigmoid(a) * _randn(g, m, d)
        elif act == "weights":
            x = 0.01 * torch.exp(0.5 * _randn(g, m, 1)) * _randn(g, m, d)
        else:
            x = _randn(g, m, d)
        out[i:i + m] = x
    return out


def _weights(g, rows, d):
    """Weight rows of unequal energy in the 4-bit form, made in slices: codes and scales."""
    codes = torch.empty((rows, d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((rows, -(-d // 512) * 16), dtype=torch.uint8, device=DEV)
    for i in range(0, rows, 8192):
        m = min(8192, rows - i)
        w = (0.02 * torch.exp(0.5 * _randn(g, m, 1)) * _randn(g, m, d)).view(m, d // 32, 32)
        q, b = _round4(w)
        code = _level(q.abs()) | ((q < 0).to(torch.uint8) << 3)
        code = code.view(m, d)
        codes[i:i + m] = code[:, 0::2] | (code[:, 1::2] << 4)
        scales[i:i + m, : d // 32] = b
    return codes, scales


def _inputs(case, seed):
    g = _generator(seed)
    n, d, op = case["n"], case["d"], case["op"]
    i = {}
    if op == "down":
        i["gu"] = _tokens(case, g, n, 2 * d)
    else:
        i["x"] = _tokens(case, g, n, d)
    if op == "norm":
        i["residual"] = (3.0 * _randn(g, n, d)).to(_type(case["dtype"]))
        i["gain"] = (1.0 + 0.2 * _randn(g, d)).to(_type(case["dtype"]))
    if op in ("linear", "down"):
        i["wq"], i["ws"] = _weights(g, case["d_out"], d)
    if op == "experts":
        e = case["experts"]
        wq, ws = _weights(g, e * case["d_out"], d)
        i["wq"], i["ws"] = wq.view(e, case["d_out"], -1), ws.view(e, case["d_out"], -1)
        logits = _randn(g, n, e) + case["skew"] * _randn(g, 1, e)
        chosen = torch.topk(logits, case["top"], dim=1).indices.reshape(-1)
        order = torch.argsort(chosen, stable=True)
        counts = torch.bincount(chosen, minlength=e)
        i["rows"] = (order // case["top"]).to(torch.int32)
        i["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        i["most"] = int(counts.max())
    return i


def prepare(case, seed):
    return {"case": case, **_inputs(case, seed)}


# ---------------------------------------------------------------------------------------- the plain form

def _power(b):
    """2^(b - 127) in 32 bits, from its bits."""
    b = b.int()
    return torch.where(b > 0, b << 23, 1 << 22).view(torch.float32)


def _round4(blocks):
    """Blocks [.., 32] in 32 bits: their values on the 4-bit grid (before the scale) and the scales' bytes."""
    a = blocks.abs().amax(-1)
    b = ((a.view(torch.int32) >> 23) - 2).clamp_min(0)                 # floor(log2 a) - 2, biased by 127
    v = blocks * _power(254 - b)[..., None]
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    q = (torch.round(m / step) * step).clamp_max(6.0)
    return torch.where(v < 0, -q, q), b.to(torch.uint8)


def _level(m):
    """The code (0 to 7) of a magnitude on the grid 0, 0.5, 1, 1.5, 2, 3, 4, 6."""
    return torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8)


def _values4(x):
    """x's values after quantization, in 32 bits."""
    blocks = x.float().view(*x.shape[:-1], -1, 32)
    q, b = _round4(blocks)
    return (q * _power(b)[..., None]).view(x.shape)


def _unpacked(codes, scales):
    """The values of a tensor in the 4-bit form, in 32 bits."""
    d = codes.shape[-1] * 2
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)         # both values of a byte
    v = pairs[codes.int()].view(*codes.shape[:-1], d // 32, 32)
    return (v * _power(scales[..., : d // 32])[..., None]).view(*codes.shape[:-1], d)


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "quantize":
        return {"values": _values4(st["x"]).to(torch.bfloat16)}
    if op == "norm":
        h = st["x"].float() + st["residual"].float()
        v = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * st["gain"].float()
        return {"h": h.to(st["x"].dtype), "values": _values4(v).to(torch.bfloat16)}
    out = _type(case["out"])
    w = _unpacked(st["wq"], st["ws"])
    if op == "linear":
        return {"y": (_values4(st["x"]) @ w.T).to(out)}
    if op == "down":
        gate, up = st["gu"].float().chunk(2, -1)
        return {"y": (_values4(gate / (1.0 + torch.exp(-gate)) * up) @ w.T).to(out)}
    # experts: each expert's rows in a slice of its own, as long as the longest, then back in order
    v = _values4(st["x"])[st["rows"].long()]
    offsets = st["offsets"].long()
    at = torch.arange(v.shape[0], device=v.device)
    e = torch.searchsorted(offsets, at, right=True) - 1
    slices = v.new_zeros(case["experts"], st["most"], case["d"])
    slices[e, at - offsets[e]] = v
    y = torch.bmm(slices, w.transpose(1, 2))
    return {"y": y[e, at - offsets[e]].to(out)}


# ----------------------------------------------------------------------------------------------- the pass

def run(st):
    if not own:
        return _plain(st)
    import paper_2603_04359_gb300 as cat
    case = st["case"]
    op = case["op"]
    if op == "quantize":
        return {"values": cat.cat_mx_dequantize(*cat.cat_mx_quantize(st["x"]), out_dtype=torch.bfloat16)}
    if op == "norm":
        xq, xs, h = cat.cat_mx_rmsnorm_quantize(st["x"], st["gain"], 1e-5, residual=st["residual"])
        return {"h": h, "values": cat.cat_mx_dequantize(xq, xs, out_dtype=torch.bfloat16)}
    out = _type(case["out"])
    if op == "linear":
        return {"y": cat.cat_mx_linear(*cat.cat_mx_quantize(st["x"]), st["wq"], st["ws"], out_dtype=out)}
    if op == "down":
        return {"y": cat.cat_mx_linear(*cat.cat_mx_swiglu_quantize(st["gu"]), st["wq"], st["ws"], out_dtype=out)}
    xq, xs = cat.cat_mx_quantize(st["x"], rows=st["rows"])
    return {"y": cat.cat_mx_linear_grouped(xq, xs, st["wq"], st["ws"], st["offsets"], out_dtype=out)}


def work(case):
    n, d, op = case["n"], case["d"], case["op"]
    item = 4 if case["dtype"] == "f32" else 2
    if op == "quantize":
        return {"bytes": n * d * (item + 2), "flops": 0}
    if op == "norm":
        return {"bytes": n * d * (3 * item + 2), "flops": 0}
    row = d / 2 + d / 32                                   # bytes of a row of weights in the 4-bit form
    out = 4 if case["out"] == "f32" else 2
    if op == "experts":
        rows, busy = n * case["top"], min(case["experts"], n * case["top"])
        return {"bytes": n * d * item + busy * case["d_out"] * row + rows * case["d_out"] * out,
                "flops": 2 * rows * d * case["d_out"]}
    read = n * d * item * (2 if op == "down" else 1)
    return {"bytes": read + case["d_out"] * row + n * case["d_out"] * out, "flops": 2 * n * d * case["d_out"]}


# ------------------------------------------------------------------------------- the definition in 64 bits

def _two_to(e):
    """2^e in float64, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid64(x):
    """Values after quantization in float64: the block's scale is the power of two two binades below its largest
    magnitude's, a value goes to the nearest of the grid's, ties to the one of even code, 6 the most."""
    x = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    a = x.abs().amax(-1, keepdim=True)
    e = (torch.frexp(a).exponent - 3).clamp_min(-127)      # a = m 2^exponent with m in [1/2, 1)
    s = _two_to(torch.where(a > 0, e, -127))
    m = x.abs() / s
    value = torch.zeros_like(m)
    for k, (lo, hi) in enumerate([(0, .5), (.5, 1), (1, 1.5), (1.5, 2), (2, 3), (3, 4), (4, 6)]):
        middle = (lo + hi) / 2
        value = torch.where((m >= middle) if k % 2 else (m > middle), hi, value)
    return (torch.sign(x) * value * s).flatten(-2)


def _weights64(codes, scales):
    low, high = (codes & 15).long(), (codes >> 4).long()
    c = torch.stack([low, high], -1).flatten(-2)
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=codes.device) / 2
    v = grid[c & 7] * (1 - 2 * (c >> 3)).double()
    b = scales[..., : c.shape[-1] // 32].long().repeat_interleave(32, -1)
    return v * _two_to(b - 127)


def exact(case, seed):
    i = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return {"values": _grid64(i["x"])}
    if op == "norm":
        h = i["x"].double() + i["residual"].double()
        v = h / torch.sqrt((h * h).sum(-1, keepdim=True) / case["d"] + 1e-5) * i["gain"].double()
        return {"h": h, "values": _grid64(v)}
    if op == "experts":
        x = _grid64(i["x"])
        edges = i["offsets"].tolist()
        y = [x[i["rows"][lo:hi].long()] @ _weights64(i["wq"][e], i["ws"][e]).T for e, (lo, hi) in enumerate(zip(edges, edges[1:]))]
        return {"y": torch.cat(y)}
    if op == "down":
        g, u = i["gu"][:, : case["d"]].double(), i["gu"][:, case["d"]:].double()
        x = _grid64(g * torch.sigmoid(g) * u)
    else:
        x = _grid64(i["x"])
    y = torch.empty((case["n"], case["d_out"]), dtype=torch.float64, device=DEV)
    for r in range(0, case["d_out"], 4096):
        y[:, r:r + 4096] = x @ _weights64(i["wq"][r:r + 4096], i["ws"][r:r + 4096]).T
    return {"y": y}
