"""The microscaled 4-bit format (MXFP4) in float64: quantization to the nearest grid value, packing, values."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
MIDDLE = (GRID[1:] + GRID[:-1]) / 2


def pitch(d):
    return -(-d // 512) * 16


def scale_bytes(x):
    """[n, d] -> the scale byte of every block of 32 (255 where a value is not finite)."""
    a = np.abs(x.reshape(x.shape[0], -1, 32)).max(-1)
    fine = np.isfinite(a)
    _, e = np.frexp(np.where(fine, a, 1.0))                      # a = m 2^e, m in [1/2, 1)
    return np.where(fine, np.where(a == 0, 0, np.maximum(e - 3 + 127, 0)), 255)


def levels(m):
    """Codes 0..7 of magnitudes: the nearest, ties to the even code, 7 the most."""
    code = np.zeros(m.shape, dtype=np.int64)
    for k, mid in enumerate(MIDDLE):
        code = np.where((m >= mid) if k % 2 else (m > mid), k + 1, code)
    return code


def quantize(x):
    """float64 [n, d] -> (codes 0..15 [n, d], scale bytes [n, d/32]); blocks with a non-finite value: 0 and 255."""
    n, d = x.shape
    b = scale_bytes(x)
    bad = (b == 255)[..., None]
    blocks = np.where(bad, 0.0, x.reshape(n, -1, 32))
    v = blocks / np.exp2(np.where(b == 255, 0, b - 127.0))[..., None]
    code = levels(np.abs(v)) | (np.signbit(v).astype(np.int64) << 3)
    return np.where(bad, 0, code).reshape(n, d), b


def pack(codes, b):
    """Codes and scale bytes as the library stores them."""
    n, d = codes.shape
    q = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
    s = np.zeros((n, pitch(d)), dtype=np.uint8)
    s[:, : d // 32] = b
    return q, s


def unpack(q, s):
    """(codes [n, d], scale bytes [n, d/32]) of the stored form."""
    d = 2 * q.shape[1]
    codes = np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], d).astype(np.int64)
    return codes, s[:, : d // 32].astype(np.int64)


def values(codes, b):
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(b == 255, np.nan, np.exp2(b - 127.0))
    return (v.reshape(*b.shape, 32) * scale[..., None]).reshape(codes.shape)
