"""The 4-bit key/value cache in float64: its layout, head norms and rotation, and attention over its pages."""
import numpy as np

import mx_reference as R


def page_bytes(page, d):
    return page * (d // 2 + d // 32)


def blank(pages, hkv, page, d, fill=0):
    return np.full((pages, 2, hkv, page_bytes(page, d)), fill, dtype=np.uint8)


def order(d, kind):
    """Byte i of a stored row is byte order[i] of the plain form: pieces of 4 bytes (keys) or 2 (values) of every block in turn."""
    piece, blocks = (4 if kind == 0 else 2), d // 32
    return np.array([16 * b + piece * p + i for p in range(16 // piece) for b in range(blocks) for i in range(piece)])


def parts(cache, page, d):
    """Views of the codes [pages, 2, hkv, page, d / 2] and the scales [pages, 2, hkv, page, d / 32]."""
    c = page * (d // 2)
    return (cache[..., :c].reshape(*cache.shape[:3], page, d // 2), cache[..., c:].reshape(*cache.shape[:3], page, d // 32))


def store(cache, page, k, v, slots):
    """Writes float64 keys and values [n, hkv, d]; slots outside the cache are left out."""
    n, hkv, d = k.shape
    rows = cache.shape[0] * page
    out = cache.copy()
    c = page * (d // 2)
    for kind, x in ((0, k), (1, v)):
        codes, b = R.quantize(x.reshape(-1, d))
        q = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)[:, order(d, kind)].reshape(n, hkv, -1)
        b = b.astype(np.uint8).reshape(n, hkv, -1)
        for i, s in enumerate(slots):
            if 0 <= s < rows:
                p, r = divmod(int(s), page)
                out[p, kind, :, r * (d // 2):(r + 1) * (d // 2)] = q[i]
                out[p, kind, :, c + r * (d // 32):c + (r + 1) * (d // 32)] = b[i]
    return out


def load(cache, page, d, slots, kind):
    """The values [m, hkv, d] of rows; zeros for slots outside the cache."""
    codes, scales = parts(cache, page, d)
    rows = cache.shape[0] * page
    slots = np.asarray(slots, dtype=np.int64)
    ok = (slots >= 0) & (slots < rows)
    s = np.where(ok, slots, 0)
    q, b = codes[s // page, kind, :, s % page], scales[s // page, kind, :, s % page]
    plain = np.empty_like(q)
    plain[..., order(d, kind)] = q
    c = np.stack([plain & 15, plain >> 4], -1).reshape(-1, d).astype(np.int64)
    v = R.values(c, b.reshape(-1, d // 32).astype(np.int64)).reshape(len(s), -1, d)
    return np.where(ok[:, None, None], v, 0.0)


def normed(x, weight, eps):
    return x if weight is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight


def turned(x, cos, sin, interleaved):
    """Heads [n, heads, d] with tables' rows cos, sin [n, rot / 2]."""
    half = cos.shape[1]
    r = 2 * half
    y = x.copy()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :half], x[..., half:r])
    u, w = a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]
    if interleaved:
        y[..., 0:r:2], y[..., 1:r:2] = u, w
    else:
        y[..., :half], y[..., half:r] = u, w
    return y


def attention(q, cache, page, table, lens, scale, offsets=None, window=0):
    """(out, a bound's parts): out [n, hq, d]; sum of weights times |v| [n, hq, d]; the largest sum of |q k| scale [n, hq]; the
    largest |v| of a row's sequence [n]; tokens a row's sequence has [n]."""
    n, hq, d = q.shape
    hkv = cache.shape[2]
    group = hq // hkv
    seqs, width = table.shape
    offsets = np.arange(seqs + 1) if offsets is None else np.clip(offsets, 0, n)
    out, mass = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    dots, vmax, count = np.zeros((n, hq)), np.zeros(n), np.zeros(n)
    for s in range(seqs):
        r0, r1 = int(offsets[s]), int(offsets[s + 1])
        have = min(max(int(lens[s]), 0), width * page)
        if r1 <= r0 or have == 0:
            continue
        t = np.arange(have)
        pages = table[s, t // page].astype(np.int64)
        there = (pages >= 0) & (pages < cache.shape[0])
        slots = np.where(there, pages * page + t % page, -1)
        k, v = load(cache, page, d, slots, 0), load(cache, page, d, slots, 1)
        fine = np.nan_to_num(np.abs(v))
        for j in range(r0, r1):
            p = int(lens[s]) - (r1 - r0) + (j - r0)
            seen = there & (t <= p) & ((t > p - window) if window else True)
            vmax[j], count[j] = fine.max(), have
            if not seen.any():
                continue
            for h in range(hkv):
                for i in range(h * group, (h + 1) * group):
                    x = k[seen, h] @ q[j, i] * scale
                    dots[j, i] = np.max(np.abs(k[seen, h]) @ np.abs(q[j, i])) * abs(scale)
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    out[j, i] = w @ v[seen, h]
                    mass[j, i] = w @ fine[seen, h]
    return out, mass, dots, vmax, count


def tolerance(out, mass, dots, vmax, count, d, bf16):
    """The bound on the kernel's error (see test_gpu_mx_attention.py)."""
    score = (2 * d + 32) * 2.0 ** -23 * dots + 2.0 ** -21
    sums = (count / 16 + 64) * 2.0 ** -23
    relative = 2 * (score + 2.0 ** -11) + sums[:, None]
    return (relative[..., None] * mass + (count * 2.0 ** -32 * vmax)[:, None, None] + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(out)
            + 2.0 ** -120)
