"""What the calls of the 4-bit key/value cache write shares no memory with what they read: refused by the library where it can tell, and by
the binding for all tensors."""
import ctypes

import pytest

import host_tensors
import paper_2603_04359_gb300 as cat
from fake_runtime import ensure_built


@pytest.fixture(scope="module")
def lib():
    ensure_built()
    return cat.load_library()


def at(i):
    return ctypes.c_void_p(0x10000000 + (i << 24))


def shared(f, args, out, size, others):
    """The call with its output `out` on the last bytes of what argument i takes, and before its first."""
    for i, bytes_ in others:
        for address in (args[i].value + bytes_ - 16, args[i].value - size + 16):
            bad = list(args)
            bad[out] = ctypes.c_void_p(address)
            assert f(*bad) == 1, (i, address)
            assert b"must not" in cat.load_library().cat_last_error()


def test_the_library_refuses_outputs_on_what_is_read(lib):
    n, hq, hkv, d, page, pages, seqs, width = 12, 4, 2, 64, 16, 6, 3, 20
    cache = pages * 2 * hkv * page * (d // 2 + d // 32)
    a = [at(0), n, hq, at(1), pages, page, hkv, d, at(2), width, at(3), seqs, at(4), 0.1, 0, 1, at(5), at(6), 1 << 20, None]
    shared(lib.cat_mx_attention, a, 16, n * hq * d * 2,
           [(0, n * hq * d * 2), (3, cache), (8, seqs * width * 4 // 16 * 16), (10, 16), (12, 16), (17, 1 << 20)])
    rot, rows = 32, 100
    r = [at(0), 1, n, hq, at(1), at(2), 1, 1e-6, at(3), at(4), at(5), rows, rot, 0, at(6), at(7), pages, page, hkv, d, at(8), None]
    shared(lib.cat_mx_rope_cache_write, r, 20, n * hq * d * 2,
           [(0, n * (hq + 2 * hkv) * d * 2), (4, d * 2), (5, d * 2), (8, 48), (9, rows * rot * 2), (10, rows * rot * 2), (14, 48), (15, cache)])


SCRIPT = """
def on_bytes(base, first, dtype, *shape):
    n = dtype.itemsize
    for a in shape:
        n *= a
    s = torch._C._construct_storage_from_data_pointer(base.data_ptr() + first, base.device, n)
    stride = [1] * len(shape)
    for i in range(len(shape) - 2, -1, -1):
        stride[i] = stride[i + 1] * shape[i + 1]
    return torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(dict(size=shape, stride=tuple(stride), dtype=dtype, storage_offset=0), s)

torch.empty = lambda shape, dtype, device: on(device.index, dtype, *shape)
cat.cat_mx_attention_workspace = lambda *a: 64
k, s, c = on(0, b, 5, 2, 64), on(0, i, 5), on(0, u, 3, 2, 2, 544)
x, cs, w = on(0, b, 5, 8 * 64), on(0, f, 100, 32), on(0, b, 64)
q, table, lens, offs, ws, o = on(0, b, 5, 4, 64), on(0, i, 3, 6), on(0, i, 3), on(0, i, 4), on(0, u, 4096), on(0, b, 5, 4, 64)
ko = on(0, b, 5, 2, 64)
calls = [
    lambda: cat.cat_mx_cache_write(on_bytes(c, 64, b, 5, 2, 64), k, s, c), lambda: cat.cat_mx_cache_write(k, on_bytes(c, 64, b, 5, 2, 64), s, c),
    lambda: cat.cat_mx_cache_write(k, k, on_bytes(c, 64, i, 5), c),
    lambda: cat.cat_mx_cache_read(c, s, 64, k=on_bytes(c, 64, b, 5, 2, 64), v=ko), lambda: cat.cat_mx_cache_read(c, s, 64, k=ko, v=on_bytes(c, 64, b, 5, 2, 64)),
    lambda: cat.cat_mx_cache_read(c, on_bytes(k, 0, i, 5), 64, k=k, v=ko), lambda: cat.cat_mx_cache_read(c, s, 64, k=k, v=k),
    lambda: cat.cat_mx_rope_cache_write(on_bytes(c, 0, b, 5, 512), 64, s, cs, cs, s, c),
    lambda: cat.cat_mx_rope_cache_write(x, 64, s, cs, cs, s, c, k_weight=on_bytes(c, 64, b, 64)),
    lambda: cat.cat_mx_rope_cache_write(x, 64, on_bytes(c, 0, i, 5), cs, cs, s, c),
    lambda: cat.cat_mx_rope_cache_write(x, 64, s, cs, cs, s, c, q=on_bytes(c, 0, b, 5, 4, 64)),
    lambda: cat.cat_mx_rope_cache_write(x, 64, s, cs, cs, s, c, q=on_bytes(x, 256, b, 5, 4, 64)),
    lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, out=q), lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, out=on_bytes(c, 64, b, 5, 4, 64)),
    lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, workspace=on_bytes(c, 64, u, 512)),
    lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, workspace=on_bytes(q, 64, u, 512)),
    lambda: cat.cat_mx_attention(q, c, on_bytes(ws, 64, i, 3, 6), lens, 0.1, offsets=offs, workspace=ws),
    lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=on_bytes(ws, 64, i, 4), workspace=ws),
    lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, out=on_bytes(ws, 0, b, 5, 4, 64), workspace=ws),
]
for n, call in enumerate(calls):
    print("shared |", n, "|", outcome(call))
# side by side is fine
both = on(0, u, 2 * 5 * 2 * 64 * 2)
print("apart | 0 |", outcome(lambda: cat.cat_mx_cache_read(c, s, 64, k=on_bytes(both, 0, b, 5, 2, 64), v=on_bytes(both, 1280, b, 5, 2, 64))))
print("apart | 1 |", outcome(lambda: cat.cat_mx_attention(q, c, table, lens, 0.1, offsets=offs, out=o, workspace=ws)))
"""


def test_the_binding_refuses_shared_memory(tmp_path):
    rows = host_tensors.run(SCRIPT, tmp_path)
    refused = [r for r in rows if r[0] == "shared"]
    assert len(refused) == 19
    for r in refused:
        assert r[2] == "ValueError" and "must not share memory" in r[3], r
    others = [r for r in rows if r[0] == "apart"]
    assert len(others) == 2
    for r in others:
        assert "must not" not in " ".join(r), r
