"""What the operators of the 4-bit key/value cache are timed on, in plain torch and as the library's calls.

A case is a dict of plain values.  ``op`` names what a pass goes through:

* ``write``: keys and values into their rows of a paged cache in the microscaled 4-bit form, and back as values.
* ``read``: rows of such a cache back as the values they stand for.
* ``rope``: a fused projection's output: the norm of each query and key head, the rotation by the token's position, keys and
  values into the cache (returned as the values they stand for there), queries out.
* ``attend``: causal attention of a ragged batch over its pages of such a cache.

``own`` chooses between the plain form and the library's calls.  The plain form is elementary operations in 32 bits; a head's
norm and rotation are in 64, as what they give is rounded to 4 bits, where one value next to a border tells.

The cache is uint8 [pages, 2 (keys, values), heads, page * (d / 2 + d / 32)]: a page of a head holds its tokens' codes (d / 2 bytes
each, value 2j in the low nibble of byte j), then their scales (a byte for 32 values, 2^(byte - 127)).  A block of 32 values is 16 bytes
of codes: in a row of keys the blocks' first 4 bytes come first, one block after another, then their second 4 bytes, and so
on; in a row of values the same with 2 bytes.
"""
import math
import random

import torch

own = False
DEV = "cuda"
EPS = 1e-6
MOST_FLOPS = 1.1e12                 # of the largest attention listed
MOST_VALUES = 8192 * 80 * 128       # of the largest projection output listed
MOST_CACHED = 64 * 8192 * 8 * 128   # keys of the largest cache listed


def listed():
    return [
        # a decode batch's keys and values: every launch counts
        dict(name="write_27", op="write", n=27, hkv=8, d=128, page=64, dtype="bf16"),
        # an encoder's float32 keys and values of a long prompt, small heads
        dict(name="write_8000_f32", op="write", n=8000, hkv=16, d=64, page=16, dtype="f32"),
        # a short prefix taken out of the cache, in float32
        dict(name="read_200_f32", op="read", n=200, hkv=8, d=128, page=16, out="f32"),
        # a long shared prefix
        dict(name="read_32768", op="read", n=32768, hkv=8, d=128, page=64, out="bf16"),
        # one token of a 4096 -> 6144 projection: latency
        dict(name="rope_1", op="rope", n=1, hq=32, hkv=8, d=128, page=64, dtype="bf16", norm=True, rot=128, pairs=False),
        # a prompt of odd length without head norms, interleaved pairs, half of each head rotated
        dict(name="rope_999_half", op="rope", n=999, hq=16, hkv=16, d=64, page=32, dtype="f32", norm=False, rot=32, pairs=True),
        # a long prompt of an 8192 wide model
        dict(name="rope_8192", op="rope", n=8192, hq=64, hkv=8, d=128, page=64, dtype="bf16", norm=True, rot=128, pairs=False),
        # a decode batch of short chats, a head of keys for each of queries
        dict(name="decode_27_short", op="attend", seqs=27, q=1, len=500, hq=12, hkv=12, d=64, page=16, window=0, ragged=True),
        # one chat with a very long context
        dict(name="decode_1_long", op="attend", seqs=1, q=1, len=131000, hq=32, hkv=8, d=128, page=64, window=0, ragged=False),
        # a busy server's decode step
        dict(name="decode_64", op="attend", seqs=64, q=1, len=8192, hq=64, hkv=8, d=128, page=64, window=0, ragged=True),
        # drafted tokens verified, sliding window
        dict(name="verify_16", op="attend", seqs=16, q=5, len=6000, hq=32, hkv=8, d=128, page=32, window=4096, ragged=True),
        # the last chunk of a long prompt
        dict(name="chunk_2048", op="attend", seqs=1, q=2048, len=32768, hq=32, hkv=8, d=128, page=64, window=0, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "rope", "rope", "attend", "attend", "attend", "attend"])
    d = rng.choice([64, 128, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128])
    hkv = rng.choice([1, 2, 4, 8, 8, 16])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op in ("write", "read"):
        n = min(_log_int(rng, 1, 32768), 32768 * 8 * 128 // (hkv * d * (2 if dtype == "f32" else 1)))
        return dict(op=op, n=n, hkv=hkv, d=d, page=page, **{"dtype" if op == "write" else "out": dtype})
    group = rng.choice([1, 2, 4, 4, 5, 8, 8, 16])
    hq = hkv * group
    if op == "rope":
        n = max(1, min(_log_int(rng, 1, 8192), MOST_VALUES // ((hq + 2 * hkv) * d * (2 if dtype == "f32" else 1))))
        return dict(op=op, n=n, hq=hq, hkv=hkv, d=d, page=page, dtype=dtype, norm=rng.random() < 0.5,
                    rot=d if rng.random() < 0.7 else d // 2, pairs=rng.random() < 0.3)
    kind = rng.choice(["decode", "decode", "verify", "prompt"])
    length = _log_int(rng, 1, 65536 if kind != "prompt" else 16384)
    seqs = min(_log_int(rng, 1, 128), max(1, MOST_CACHED // (length * hkv * d)))
    q = 1
    if kind == "verify":
        q = rng.randint(2, 16)
    elif kind == "prompt":
        seqs = min(seqs, 6)
        q = length if rng.random() < 0.5 else _log_int(rng, 1, length)
    # the plain form's scores are held whole
    while 4 * d * hq * seqs * q * length > MOST_FLOPS or hq * seqs * q * length > 2 ** 31:
        q, length = max(1, q * 2 // 3), max(1, length * 2 // 3)
    return dict(op="attend", seqs=seqs, q=q, len=length, hq=hq, hkv=hkv, d=d, page=page,
                window=_log_int(rng, 1, max(2, length)) if rng.random() < 0.25 else 0, ragged=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 31)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _batch(case):
    """Lengths of the sequences and of their queries: the case's own, or ragged ones up to them (a slot of a batch may be idle)."""
    rng = random.Random(case["len"] * 131 + case["seqs"])
    lens, rows = [case["len"]] * case["seqs"], [case["q"]] * case["seqs"]
    if case["ragged"]:
        for s in range(1, case["seqs"]):
            lens[s] = 0 if s % 16 == 15 else max(1, int(case["len"] * rng.uniform(0.05, 1.0)))
            if case["q"] > 16:
                rows[s] = max(1, min(lens[s], int(case["q"] * rng.uniform(0.05, 1.0))))
    return lens, rows


def _cache(pages, hkv, page, d):
    return torch.zeros((pages, 2, hkv, page * (d // 2 + d // 32)), dtype=torch.uint8, device=DEV)


def _head_channels(g, hkv, d):
    """Factors of a head's channels: keys have a few much larger ones."""
    f = 1.0 + 0.3 * _randn(g, hkv, d).abs()
    f[:, : max(1, d // 64)] *= 8.0
    return f


def _slots(g, case, pages):
    """Rows of the cache for a case's tokens: runs of page length in pages that lie anywhere."""
    page = case["page"]
    order = torch.randperm(pages, generator=g, device=DEV)[: -(-case["n"] // page)]
    at = torch.arange(case["n"], device=DEV)
    return (order[at // page] * page + at % page).to(torch.int32)


def _angles(case):
    """cos and sin [positions, rot / 2] in 32 bits, of angles in 64."""
    half = case["rot"] // 2
    freq = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    a = torch.arange(32768, dtype=torch.float64, device=DEV)[:, None] * freq
    return torch.cos(a).float(), torch.sin(a).float()


def _fill(g, cache, case, slots):
    """Random keys and values into the rows of the cache that `slots` names, made in slices."""
    hkv, d = case["hkv"], case["d"]
    factors = _head_channels(g, hkv, d)
    step = max(1, 2 ** 26 // (hkv * d))
    for i in range(0, len(slots), step):
        at = slots[i:i + step]
        _store(cache, case, at, _randn(g, len(at), hkv, d) * factors, _randn(g, len(at), hkv, d) + 0.25)


def _inputs(case, seed):
    g = _generator(seed)
    op, hkv, d, page = case["op"], case["hkv"], case["d"], case["page"]
    i = {}
    if op == "attend":
        lens, rows = _batch(case)
        widest = max(1, -(-max(lens) // page))
        pages = [-(-n // page) for n in lens]
        order = torch.randperm(sum(pages) + 3, generator=g, device=DEV).to(torch.int32)
        table = torch.zeros((case["seqs"], widest), dtype=torch.int32, device=DEV)
        counts = torch.tensor(pages, device=DEV)
        table[torch.arange(widest, device=DEV) < counts[:, None]] = order[: sum(pages)]
        i["cache"] = _cache(sum(pages) + 3, hkv, page, d)
        i["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        i["table"] = table
        at = torch.arange(widest * page, device=DEV)
        slots = (table[:, at // page] * page + at % page)[at < i["lens"][:, None]]
        _fill(g, i["cache"], case, slots)
        i["offsets"] = torch.tensor([0] + rows, device=DEV).cumsum(0).to(torch.int32)
        i["most"] = max(rows)
        i["queries"] = (1.5 * _randn(g, sum(rows), case["hq"], d)).to(torch.bfloat16)
        return i
    pages = -(-case["n"] // page) + 5
    i["cache"] = _cache(pages, hkv, page, d)
    i["slots"] = _slots(g, case, pages)
    if op == "read":
        _fill(g, i["cache"], case, i["slots"])
    elif op == "write":
        i["keys"] = (_randn(g, case["n"], hkv, d) * _head_channels(g, hkv, d)).to(_type(case["dtype"]))
        i["values"] = _randn(g, case["n"], hkv, d).to(_type(case["dtype"]))
    else:
        heads = case["hq"] + 2 * hkv
        i["qkv"] = (_randn(g, case["n"], heads, 1).exp() * _randn(g, case["n"], heads, d)).view(case["n"], heads * d).to(_type(case["dtype"]))
        i["cos"], i["sin"] = _angles(case)
        i["positions"] = torch.randint(0, 32768, (case["n"],), generator=g, device=DEV, dtype=torch.int32)
        if case["norm"]:
            i["gain_q"] = (1.0 + 0.2 * _randn(g, d)).to(_type(case["dtype"]))
            i["gain_k"] = _head_channels(g, 1, d)[0].to(_type(case["dtype"]))
    return i


def prepare(case, seed):
    return {"case": case, **_inputs(case, seed)}


# ---------------------------------------------------------------------------------------- the plain form

def _power(b):
    """2^(b - 127) in 32 bits, from its bits."""
    b = b.int()
    return torch.where(b > 0, b << 23, 1 << 22).view(torch.float32)


def _quantized(x):
    """Rows [.., d] of 32 or 64 bits: codes, two a byte, [.., d / 2] and scales [.., d / 32]."""
    blocks = x.unflatten(-1, (-1, 32))
    a = blocks.abs().amax(-1)
    e = torch.frexp(a).exponent - 1                                              # floor(log2 a)
    b = torch.where(a > 0, (e + 125).clamp_min(0), torch.zeros_like(e))
    v = blocks * _power(254 - b)[..., None].to(x.dtype)
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).to(x.dtype)
    m = (torch.round(m / step) * step).clamp_max(6.0)
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), b.to(torch.uint8)


def _views(cache, d, page):
    """Codes [pages, 2, heads, page, d / 2] and scales [pages, 2, heads, page, d / 32] of a cache."""
    codes = page * (d // 2)
    return cache[..., :codes].unflatten(-1, (page, d // 2)), cache[..., codes:].unflatten(-1, (page, d // 32))


def _store(cache, case, slots, keys, values):
    d, page = case["d"], case["page"]
    codes, scales = _views(cache, d, page)
    p, at = slots.long() // page, slots.long() % page
    for kind, x, parts in ((0, keys, 4), (1, values, 8)):
        c, s = _quantized(x)
        codes[:, kind][p, :, at] = c.unflatten(-1, (d // 32, parts, 16 // parts)).transpose(-3, -2).flatten(-3)
        scales[:, kind][p, :, at] = s


def _values(codes, scales, kind):
    """The values of rows of keys (kind 0) or values (1), in 32 bits."""
    d, parts = 2 * codes.shape[-1], 4 if kind == 0 else 8
    codes = codes.unflatten(-1, (parts, d // 32, 16 // parts)).transpose(-3, -2).flatten(-3)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)         # both values of a byte
    v = pairs[codes.int()].flatten(-2).unflatten(-1, (d // 32, 32))
    return (v * _power(scales)[..., None]).flatten(-2)


def _rows(cache, case, slots):
    """Keys and values of the rows that `slots` names, [rows, heads, d] in 32 bits."""
    codes, scales = _views(cache, case["d"], case["page"])
    p, at = slots.long() // case["page"], slots.long() % case["page"]
    return [_values(codes[:, k][p, :, at], scales[:, k][p, :, at], k) for k in (0, 1)]


def _normed(x, gain):
    if gain is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.double()


def _turned(x, cos, sin, pairs):
    """The first channels of heads [n, heads, d] rotated, in pairs of neighbours or of both halves."""
    r = 2 * cos.shape[-1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if pairs else (x[..., : r // 2], x[..., r // 2: r])
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _attended(st, case):
    lens, offsets, page, d, hkv = st["lens"].long(), st["offsets"].long(), case["page"], case["d"], case["hkv"]
    seqs, most = case["seqs"], st["most"]
    codes, scales = _views(st["cache"], d, page)
    k, v = (_values(codes[:, i][st["table"].long()], scales[:, i][st["table"].long()], i).transpose(1, 2).flatten(2, 3) for i in (0, 1))
    total = k.shape[2]                                                             # keys [seqs, hkv, total, d]
    count = offsets[1:] - offsets[:-1]
    j = torch.arange(most, device=lens.device)
    real = j < count[:, None]                                                      # [seqs, most]
    q = st["queries"].new_zeros((seqs, most, case["hq"], d), dtype=torch.float32)
    q[real] = st["queries"].float()
    q = q.unflatten(2, (hkv, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)             # [seqs, hkv, group * most, d]
    last = (lens - count)[:, None] + j                                             # position of each query
    t = torch.arange(total, device=lens.device)
    seen = (t <= last[..., None]) & (t < lens[:, None, None])
    if case["window"]:
        seen &= t > last[..., None] - case["window"]
    scores = torch.matmul(q, k.transpose(2, 3)).unflatten(2, (-1, most)) * d ** -0.5
    scores = scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-1e30)
    p = scores.sub_(top).exp_()
    sums = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (-1, most)) / torch.where(sums > 0, sums, torch.ones_like(sums))
    return out.permute(0, 3, 1, 2, 4).flatten(2, 3)[real].to(torch.bfloat16)


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "attend":
        return {"out": _attended(st, case)}
    if op == "read":
        keys, values = _rows(st["cache"], case, st["slots"])
        return {"keys": keys.to(_type(case["out"])), "values": values.to(_type(case["out"]))}
    out = {}
    if op == "write":
        keys, values = st["keys"].float(), st["values"].float()
    else:
        hq, hkv = case["hq"], case["hkv"]
        q, keys, values = st["qkv"].double().unflatten(1, (-1, case["d"])).split([hq, hkv, hkv], 1)
        at = st["positions"].long()
        cos, sin = st["cos"][at][:, None].double(), st["sin"][at][:, None].double()
        out["queries"] = _turned(_normed(q, st.get("gain_q")), cos, sin, case["pairs"]).to(torch.bfloat16)
        keys = _turned(_normed(keys, st.get("gain_k")), cos, sin, case["pairs"])
    _store(st["cache"], case, st["slots"], keys, values)
    keys, values = _rows(st["cache"], case, st["slots"])
    return {**out, "keys": keys.to(torch.bfloat16), "values": values.to(torch.bfloat16)}


# ----------------------------------------------------------------------------------------------- the pass

def run(st):
    if not own:
        return _plain(st)
    import paper_2603_04359_gb300 as cat
    case = st["case"]
    op, d = case["op"], case["d"]
    if op == "attend":
        return {"out": cat.cat_mx_attention(st["queries"], st["cache"], st["table"], st["lens"], d ** -0.5, offsets=st["offsets"],
                                            window=case["window"])}
    out = {}
    if op == "write":
        cat.cat_mx_cache_write(st["keys"], st["values"], st["slots"], st["cache"])
    elif op == "rope":
        out["queries"] = cat.cat_mx_rope_cache_write(st["qkv"], d, st["positions"], st["cos"], st["sin"], st["slots"], st["cache"],
                                                     q_weight=st.get("gain_q"), k_weight=st.get("gain_k"), eps=EPS,
                                                     interleaved=case["pairs"])
    keys, values = cat.cat_mx_cache_read(st["cache"], st["slots"], d, out_dtype=_type(case.get("out", "bf16")))
    return {**out, "keys": keys, "values": values}


def work(case):
    op, hkv, d = case["op"], case["hkv"], case["d"]
    token = 2 * hkv * (d // 2 + d // 32)                   # bytes of a token's keys and values in the 4-bit form
    if op == "attend":
        lens, rows = _batch(case)
        tokens = pairs = 0
        for n, q in zip(lens, rows):
            first = max(0, n - q + 1 - case["window"]) if case["window"] else 0
            tokens += max(0, n - first)
            for j in range(q):
                p = n - q + j
                pairs += max(0, min(p + 1, case["window"] or p + 1))
        return {"bytes": tokens * token + 4 * sum(rows) * case["hq"] * d, "flops": 4 * d * case["hq"] * pairs}
    n = case["n"]
    if op == "read":
        return {"bytes": n * (token + 2 * hkv * d * (4 if case["out"] == "f32" else 2)), "flops": 0}
    item = 4 if case["dtype"] == "f32" else 2
    if op == "write":                                      # read, written as codes, read back as 16 bits
        return {"bytes": n * (2 * hkv * d * (item + 2) + token), "flops": 0}
    return {"bytes": n * ((case["hq"] + 2 * hkv) * d * (item + 2) + token + 4 * case["rot"]), "flops": 0}


# ------------------------------------------------------------------------------- the definition in 64 bits

def _grid64(x):
    """Values after quantization in float64: the block's scale is the power of two two binades below its largest
    magnitude's, a value goes to the nearest of the grid's, ties to the one of even code, 6 the most."""
    x = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    a = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(a))
    e = torch.where(torch.exp2(e) > a, e - 1, torch.where(torch.exp2(e + 1) <= a, e + 1, e))
    s = torch.exp2(torch.where(a > 0, (e - 2).clamp_min(-127), -127.0))
    m = x.abs() / s
    value = torch.zeros_like(m)
    for k, (lo, hi) in enumerate([(0, .5), (.5, 1), (1, 1.5), (1.5, 2), (2, 3), (3, 4), (4, 6)]):
        middle = (lo + hi) / 2
        value = torch.where((m >= middle) if k % 2 else (m > middle), hi, value)
    return (torch.sign(x) * value * s).flatten(-2)


def _row64(page_bytes, at, d, page, kind):
    """The values in float64 of tokens `at` of a head's pages, page_bytes [tokens, bytes of a page]: each value's byte by its place."""
    i = torch.arange(d, device=at.device)
    j = i // 2                                             # the byte in the plain order
    unit = 4 if kind == 0 else 2
    place = ((j % 16) // unit) * (unit * (d // 32)) + (j // 16) * unit + j % unit
    byte = page_bytes.gather(1, at[:, None] * (d // 2) + place).long()
    code = torch.where(i % 2 == 0, byte & 15, byte >> 4)
    scale = page_bytes.gather(1, page * (d // 2) + at[:, None] * (d // 32) + i // 32).double()
    e, f = (code & 7) // 2, (code & 1).double()
    size = torch.where(e == 0, f / 2, torch.exp2(e.double() - 1) * (1 + f / 2))
    return size * (1 - 2 * (code >> 3)).double() * torch.exp2(scale - 127)


def _attend64(case, i):
    lens, rows = _batch(case)
    d, page, group = case["d"], case["page"], case["hq"] // case["hkv"]
    out, first = [], 0
    for s, (n, q) in enumerate(zip(lens, rows)):
        mine = i["queries"][first:first + q].double()
        first += q
        o = torch.zeros_like(mine)
        out.append(o)
        if n == 0:
            continue
        t = torch.arange(n, device=DEV)
        pages = i["table"][s].long()[t // page]
        p = n - q + torch.arange(q, device=DEV)[:, None]
        hidden = (t > p) | (p < 0)
        if case["window"]:
            hidden |= t <= p - case["window"]
        for h in range(case["hkv"]):
            k = _row64(i["cache"][pages, 0, h], t % page, d, page, 0)
            v = _row64(i["cache"][pages, 1, h], t % page, d, page, 1)
            for u in range(h * group, (h + 1) * group):
                x = (mine[:, u] @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                o[:, u] = torch.nan_to_num(torch.softmax(x, -1)) @ v
    return torch.cat(out)


def exact(case, seed):
    i = _inputs(case, seed)
    op, d, page, hkv = case["op"], case["d"], case["page"], case["hkv"]
    if op == "attend":
        return {"out": _attend64(case, i)}
    if op == "read":
        s = i["slots"].long()
        keys, values = (torch.stack([_row64(i["cache"][s // page, k, h], s % page, d, page, k) for h in range(hkv)], 1) for k in (0, 1))
        return {"keys": keys, "values": values}
    if op == "write":
        return {"keys": _grid64(i["keys"]), "values": _grid64(i["values"])}
    x = i["qkv"].double().view(case["n"], -1, d)
    hq = case["hq"]
    if case["norm"]:
        mean = (x * x).sum(-1, keepdim=True) / d
        gains = torch.cat([i["gain_q"].double().expand(hq, d), i["gain_k"].double().expand(hkv, d)])
        x = torch.cat([x[:, :hq + hkv] / torch.sqrt(mean[:, :hq + hkv] + EPS) * gains, x[:, hq + hkv:]], 1)
    # a rotation is a product with a complex number of the tables' parts
    at, half = i["positions"].long(), case["rot"] // 2
    z = torch.complex(i["cos"][at].double(), i["sin"][at].double())[:, None]
    turn = x[:, :hq + hkv, :case["rot"]]
    turn = turn.unflatten(-1, (half, 2)) if case["pairs"] else turn.unflatten(-1, (2, half)).transpose(-1, -2)
    w = torch.view_as_real(torch.view_as_complex(turn.contiguous()) * z)
    turn = w.flatten(-2) if case["pairs"] else w.transpose(-1, -2).flatten(-2)
    qk = torch.cat([turn, x[:, :hq + hkv, case["rot"]:]], -1)
    return {"queries": qk[:, :hq], "keys": _grid64(qk[:, hq:]), "values": _grid64(x[:, hq + hkv:])}
