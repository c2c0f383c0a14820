"""The 4-bit key/value cache without a GPU: the reference's layout, what the library and the binding refuse, what is launched."""
import ctypes

import numpy as np
import pytest
import torch

import host_tensors
import mx_cache_reference as C
import mx_reference as R
import paper_2603_04359_gb300 as cat
from fake_runtime import FakeRuntime, ensure_built

P, BAD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)
A = 0x10 << 40          # an address that holds nothing


@pytest.fixture(scope="module")
def lib():
    ensure_built()
    return cat.load_library()


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 32)])
def test_reference_layout(d, page):
    """A row's pieces by the format's words: piece p of block b of keys is 4 bytes at 4 (p d/32 + b), of values 2 at 2 (..)."""
    rng = np.random.default_rng(d)
    k, v = rng.standard_normal((3, 2, d)), rng.standard_normal((3, 2, d))
    slots = [5, page + 1, -1]
    cache = C.store(C.blank(2, 2, page, d), page, k, v, slots)
    codes, b = R.quantize(k[1])
    plain = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
    row = cache[1, 0, :, (d // 2):2 * (d // 2)]
    for blk in range(d // 32):
        for p in range(4):
            at = 4 * (p * (d // 32) + blk)
            np.testing.assert_array_equal(row[:, at:at + 4], plain[:, 16 * blk + 4 * p:16 * blk + 4 * p + 4])
    np.testing.assert_array_equal(cache[1, 0, :, page * (d // 2) + d // 32:page * (d // 2) + 2 * (d // 32)], b)
    for kind, x in ((0, k), (1, v)):
        got = C.load(cache, page, d, [5, page + 1, 7, 99999], kind)
        c, s = R.quantize(x.reshape(-1, d))
        np.testing.assert_array_equal(got[:2], R.values(c, s).reshape(3, 2, d)[:2])
        assert not got[2:].any()


def test_page_bytes(lib):
    for page in (0, 8, 15, 16, 24, 64, 1024, 2048, -16):
        for d in (0, 32, 64, 96, 128, 256, 512):
            want = page * (d // 2 + d // 32) if d in (64, 128, 256) and page in (16, 64, 1024) else 0
            assert lib.cat_mx_cache_page_bytes(page, d) == cat.cat_mx_cache_page_bytes(page, d) == want
    with pytest.raises(ValueError):
        cat.cat_mx_cache(2, 1, 24, 64, device="cpu")
    assert cat.cat_mx_cache(2, 3, 16, 64, device="cpu").shape == (2, 2, 3, 544)


def test_refusals(lib):
    """Invalid calls are refused on the host, before anything touches CUDA."""
    # (k, v, dtype, n, slots, cache, pages, page, hkv, d, stream)
    w = lib.cat_mx_cache_write
    good = [P, P, 1, 4, P, P, 2, 16, 2, 64, None]

    def refused(f, good, status, **at):
        args = list(good)
        for i, v in at.items():
            args[int(i[1:])] = v
        assert f(*args) == status, at
    for i, v in ((2, 2), (0, None), (1, None), (4, None), (5, None)):
        refused(w, good, 1, **{f"_{i}": v})
    for i, v in ((3, -1), (3, 1 << 31), (6, -1), (6, 1 << 27), (7, 8), (7, 48), (7, 2048), (8, 0), (8, 65537), (9, 96), (9, 512)):
        refused(w, good, 2, **{f"_{i}": v})
    for i in (0, 1, 4, 5):
        refused(w, good, 3, **{f"_{i}": BAD})
    refused(w, good, 0, _3=0, _0=None, _1=None, _4=None)
    # (cache, pages, page, hkv, d, slots, m, out_dtype, k, v, stream)
    r = lib.cat_mx_cache_read
    good = [P, 2, 16, 2, 64, P, 4, 0, P, P, None]
    for i, v in ((7, 3), (0, None), (5, None), (8, None), (9, None)):
        refused(r, good, 1, **{f"_{i}": v})
    for i, v in ((1, -1), (2, 0), (3, 0), (4, 63), (6, -1)):
        refused(r, good, 2, **{f"_{i}": v})
    for i in (0, 5, 8, 9):
        refused(r, good, 3, **{f"_{i}": BAD})
    refused(r, good, 0, _6=0)
    # (qkv, dtype, n, hq, q_weight, k_weight, weight_dtype, eps, positions, cos, sin, table_rows, rot, interleaved, slots, cache,
    #  pages, page, hkv, d, q_out, stream)
    f = lib.cat_mx_rope_cache_write
    good = [P, 1, 4, 4, P, P, 0, 1e-6, P, P, P, 100, 64, 0, P, P, 2, 16, 2, 64, P, None]
    for i, v in ((1, 2), (6, 5), (7, -1.0), (7, float("nan")), (7, float("inf")), (13, 2), (0, None), (8, None), (9, None), (10, None),
                 (14, None), (15, None), (20, None)):
        refused(f, good, 1, **{f"_{i}": v})
    for i, v in ((2, -1), (2, 1 << 31), (3, 0), (3, 65537), (11, -1), (12, 0), (12, 8), (12, 24), (12, 80), (16, -1), (17, 17), (18, 0), (19, 32)):
        refused(f, good, 2, **{f"_{i}": v})
    for i in (0, 4, 5, 8, 9, 10, 14, 15, 20):
        refused(f, good, 3, **{f"_{i}": BAD})
    refused(f, good, 0, _2=0, _0=None)
    # (q, n, hq, cache, pages, page, hkv, d, table, width, lens, seqs, offsets, scale, window, out_dtype, out, ws, bytes, stream)
    a = lib.cat_mx_attention
    good = [P, 4, 4, P, 2, 16, 2, 64, P, 3, P, 4, None, 0.1, 0, 1, P, P, 1 << 40, None]
    for i, v in ((13, float("nan")), (13, float("inf")), (15, 2), (0, None), (3, None), (8, None), (10, None), (16, None)):
        refused(a, good, 1, **{f"_{i}": v})
    for i, v in ((1, -1), (1, 1 << 30), (1, 3), (2, 3), (2, 0), (4, -1), (5, 12), (6, 0), (7, 65), (9, -1), (9, 1 << 28), (11, -1),
                 (11, 65537), (14, -1), (14, 1 << 31)):
        refused(a, good, 2, **{f"_{i}": v})
    for i in (0, 3, 8, 10, 12, 16, 17):
        refused(a, good, 3, **{f"_{i}": BAD})
    refused(a, good, 0, _1=0, _11=0)
    # outputs that overlap what is read while they are written, or one another
    far, near = ctypes.c_void_p(0x10000 + 4 * 4 * 64 * 2), ctypes.c_void_p(0x10000 + 4 * 4 * 64 * 2 - 16)
    for out in (P, near):
        refused(a, good, 1, _16=out)
        assert b"overlap" in lib.cat_last_error()
    near_v = ctypes.c_void_p(0x10000 + 4 * 2 * 64 * 4 - 16)
    for v in (P, near_v):
        refused(r, [P, 2, 16, 2, 64, P, 4, 0, P, P, None], 1, _9=v)
        assert b"overlap" in lib.cat_last_error()
    refused(f, [P, 1, 4, 4, P, P, 0, 1e-6, P, P, P, 100, 64, 0, P, P, 2, 16, 2, 64, P, None], 1, _20=ctypes.c_void_p(0x10000 + 4 * 8 * 64 * 2 - 16))
    if not torch.cuda.is_available():                    # (those beside one another are not refused for that)
        assert a(*(good[:16] + [far] + good[17:])) != 1 or b"overlap" not in lib.cat_last_error()
    for bad in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 3, 2, 64), (1, 1, 4, 0, 64), (1, 1, 4, 2, 96)):
        assert lib.cat_mx_attention_workspace(*bad) == 0


SCRIPT = """
torch.empty = lambda shape, dtype, device: on(device.index, dtype, *shape)
cat.cat_mx_attention_workspace = lambda *a: 64
native = cat._calls()
k, kf, s, c = on(0, b, 5, 2, 64), on(0, f, 5, 2, 64), on(0, i, 5), on(0, u, 3, 2, 2, 544)
other = on(1, u, 3, 2, 2, 544)
x, cs = on(0, b, 5, 8 * 64), on(0, f, 100, 32)
w, wf = on(0, b, 64), on(0, f, 64)
q, table, lens, offs = on(0, b, 5, 4, 64), on(0, i, 3, 6), on(0, i, 3), on(0, i, 4)
valid = {
    "cache_write": [(k, k, s, c), (kf, kf, s, c)],
    "cache_read": [(c, s, 64, None), (c, s, 64, b), (c, on(0, i, 9), 64, f)],
    "rope_cache_write": [(x, 64, s, cs, cs, s, c, w, w, 1e-6, False), (x, 64, s, cs, cs, s, c, None, wf, 0.0, True),
                         (on(0, f, 5, 512), 64, s, cs, cs, s, c, None, None, 1, 0)],
    "attention": [(q, c, table, lens, 0.1, offs, 0, None), (q, c, table, lens, 1, offs, 7, f),
                  (q, c, on(0, i, 5, 6), on(0, i, 5), 0.1, None, 0, b)],
}
others = {
    "cache_write": [(on(0, h, 5, 2, 64), on(0, h, 5, 2, 64), s, c), (k, kf, s, c), (k, k, on(0, l, 5), c), (k, k, on(0, i, 4), c),
                    (k, k, s, other), (k, k, s, on(0, u, 3, 2, 1, 544)), (k, k, s, on(0, u, 3, 1, 2, 544)), (k, k, s, on(0, u, 3, 2, 2, 540)),
                    (k, k, s, on(0, u, 3, 2, 2, 272)), (k, k, s, on(0, f, 3, 2, 2, 544)), (k, on(1, b, 5, 2, 64), s, c),
                    (k, on(0, b, 4, 2, 64), s, c), (on(0, b, 5, 2, 96), on(0, b, 5, 2, 96), s, c), (k, k, on(1, i, 5), c), (k, k, [1], c),
                    (on(0, b, 5, 2, 64, stride=(512, 64, 1)), k, s, c), (on(0, b, 5, 128), on(0, b, 5, 128), s, c),
                    (on(1, b, 5, 2, 64), on(1, b, 5, 2, 64), on(1, i, 5), other), (torch.zeros(5, 2, 64), torch.zeros(5, 2, 64), s, c)],
    "cache_read": [(c, s, 128, None), (c, s, 96, None), (c, s, 64, h), (c, on(0, l, 5), 64, None), (c, on(1, i, 5), 64, None),
                   (c, on(0, i, 2, 5), 64, None), (on(0, f, 3, 2, 2, 544), s, 64, None), (other, on(1, i, 5), 64, None),
                   (on(0, u, 3, 2, 544), s, 64, None), (c, [0], 64, None), (on(0, u, 3, 2, 2, 544, stride=(4096, 1088, 544, 1)), s, 64, None)],
    "rope_cache_write": [(on(0, h, 5, 512), 64, s, cs, cs, s, c, w, w, 1e-6, False), (on(0, b, 5, 500), 64, s, cs, cs, s, c, w, w, 1e-6, False),
                         (on(0, b, 5, 256), 64, s, cs, cs, s, c, w, w, 1e-6, False), (x, 128, s, cs, cs, s, c, w, w, 1e-6, False),
                         (x, 64, on(0, i, 4), cs, cs, s, c, w, w, 1e-6, False), (x, 64, s, on(0, b, 100, 32), cs, s, c, w, w, 1e-6, False),
                         (x, 64, s, cs, on(0, f, 99, 32), s, c, w, w, 1e-6, False), (x, 64, s, cs, cs, on(0, l, 5), c, w, w, 1e-6, False),
                         (x, 64, s, cs, cs, s, other, w, w, 1e-6, False), (x, 64, s, cs, cs, s, c, w, wf, 1e-6, False),
                         (x, 64, s, cs, cs, s, c, on(0, b, 32), None, 1e-6, False), (x, 64, s, cs, cs, s, c, on(0, h, 64), None, 1e-6, False),
                         (x, 64, s, cs, cs, s, c, w, on(1, b, 64), 1e-6, False), (x, 64, s, on(0, f, 3200), on(0, f, 3200), s, c, w, w, 1e-6, False),
                         (on(0, b, 5, 512, stride=(1024, 1)), 64, s, cs, cs, s, c, w, w, 1e-6, False), (x, 64, s, cs, cs, s, c, w, w, "a", False)],
    "attention": [(on(0, f, 5, 4, 64), c, table, lens, 0.1, offs, 0, None), (on(0, h, 5, 4, 64), c, table, lens, 0.1, offs, 0, None),
                  (q, other, table, lens, 0.1, offs, 0, None), (q, on(0, u, 3, 2, 2, 1088 * 3), table, lens, 0.1, offs, 0, None),
                  (q, c, on(0, l, 3, 6), lens, 0.1, offs, 0, None), (q, c, on(0, i, 18), lens, 0.1, offs, 0, None),
                  (q, c, on(1, i, 3, 6), lens, 0.1, offs, 0, None), (q, c, table, on(0, i, 4), 0.1, offs, 0, None),
                  (q, c, table, on(0, l, 3), 0.1, offs, 0, None), (q, c, table, lens, 0.1, on(0, i, 3), 0, None),
                  (q, c, table, lens, 0.1, on(0, l, 4), 0, None), (q, c, table, lens, 0.1, offs, 0, h), (q, c, table, lens, 0.1, [0], 0, None),
                  (on(0, b, 5, 4, 96), c, table, lens, 0.1, offs, 0, None), (on(0, b, 5, 4, 64, stride=(512, 64, 1)), c, table, lens, 0.1, offs, 0, None),
                  (on(1, b, 5, 4, 64), other, on(1, i, 3, 6), on(1, i, 3), 0.1, on(1, i, 4), 0, None), (on(0, b, 20, 64), c, table, lens, 0.1, offs, 0, None)],
}
python = {"cache_write": cat.cat_mx_cache_write, "cache_read": lambda c, s, d, t: cat.cat_mx_cache_read(c, s, d, out_dtype=t),
          "rope_cache_write": cat.cat_mx_rope_cache_write,
          "attention": lambda q, c, t, n, s, o, w, y: cat.cat_mx_attention(q, c, t, n, s, offsets=o, window=w, out_dtype=y)}
for kind, sets in (("valid", valid), ("other", others)):
    for name, calls in sets.items():
        for n, a in enumerate(calls):
            print(kind, "|", name, n, "| compiled |", outcome(lambda: getattr(native, name)(*a)))
            print(kind, "|", name, n, "| python |", outcome(lambda: python[name](*a)))
"""


@pytest.fixture(scope="module")
def outcomes(tmp_path_factory):
    return host_tensors.run(SCRIPT, tmp_path_factory.mktemp("cache_refusals"))


def test_valid_calls_pass_the_checks(outcomes):
    """(On a machine without a GPU they end at the first allocation or launch.)"""
    rows = [r for r in outcomes if r[0] == "valid"]
    assert len(rows) == 22
    for r in rows:
        assert r[3] in ("AcceleratorError", "CatError") or r[3:] == ["returned", "int"], r


def test_other_calls_pass_neither(outcomes):
    rows = [r for r in outcomes if r[0] == "other"]
    assert len(rows) == 126
    for r in rows:
        if r[2] == "compiled":
            assert (r[3], r[4]) == ("returned", "None") or r[3] == "TypeError", r
        else:
            assert r[3] in ("ValueError", "TypeError", "ArgumentError"), r


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeRuntime(tmp_path_factory.mktemp("fake_cache"))


FAR = 1 << 46             # of outputs that must not overlap what is read


def cache_calls(lib):
    for d in (64, 128, 256):
        for dtype in (0, 1):
            for n, hkv, page in ((1, 1, 16), (27, 8, 64), (100000, 5, 1024)):
                yield "cat_mx_cache_write", A, A, dtype, n, A, A, 1000, page, hkv, d, None
                yield "cat_mx_cache_read", A, 1000, page, hkv, d, A, n, dtype, A, FAR, None
                for rot in (16, 32, 64):
                    for interleaved in (0, 1):
                        yield ("cat_mx_rope_cache_write", A, dtype, n, 4 * hkv, A, None, 1, 1e-6, A, A, A, 999, rot * (d // 64), interleaved,
                               A, A, 1000, page, hkv, d, FAR, None)
            for n, seqs, hq, hkv in ((1, 1, 1, 1), (64, 64, 64, 8), (100, 20, 32, 8), (5000, 1, 16, 16), (300, 300, 128, 1)):
                need = lib.cat_mx_attention_workspace(n, seqs, hq, hkv, d)
                for offsets in (None, A):
                    if offsets or n == seqs:
                        yield ("cat_mx_attention", A, n, hq, A, 1000, 64, hkv, d, A, 50, A, seqs, offsets, 0.1, 0, dtype, FAR, A, need, None)


def test_every_launch_is_allowed_on_every_device(fake):
    first, second = [], []
    for found, device in ((first, 2), (second, 6)):
        fake.device(device)
        for name, *args in cache_calls(fake.lib):
            launches = fake.call(name, *args)
            assert 1 <= len(launches) <= (1 if name != "cat_mx_attention" else 4), (name, args)
            found += launches
    fake.device(0)
    assert [x._replace(device=0) for x in first] == [x._replace(device=0) for x in second]
    assert {x.device for x in second} == {6}


def test_a_workspace_that_is_too_small_is_refused(fake):
    need = fake.lib.cat_mx_attention_workspace(4, 4, 8, 2, 128)
    assert need > 0
    args = [A, 4, 8, A, 10, 64, 2, 128, A, 50, A, 4, None, 0.1, 0, 1, FAR]
    assert fake.lib.cat_mx_attention(*args, A, need - 1, None) == 2
    assert fake.lib.cat_mx_attention(*args, None, need, None) == 2
    assert fake.lib.cat_mx_attention(*args, A, need, None) == 0
