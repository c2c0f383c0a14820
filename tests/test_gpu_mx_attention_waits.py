"""Attention's waits that run out (a bound of 1 ns): each kernel drains its copies and MMAs, frees its tensor memory, returns and says so;
the next calls give what they gave before.  (Large enough for pieces of many steps, whose copies are not all there when they are wanted.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

cat = pytest.importorskip("paper_2603_04359_gb300")
DEV = "cuda"
CAT_ERR_TIMEOUT = 7


def call(lens, rows, hq, hkv, d, page=64, seed=51):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + d)
    counts = [-(-n // page) for n in lens]
    pages, width = sum(counts), max(counts)
    if sum(rows) > len(rows):                            # (room behind: long rows go by tiles)
        width += 2 ** 22 // (sum(rows) * hq * page)
    cache = torch.randint(0, 256, (pages, 2, hkv, cat.cat_mx_cache_page_bytes(page, d)), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8)
    cache[..., page * (d // 2):] = cache[..., page * (d // 2):] % 8 + 120
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = torch.arange(at, at + c, dtype=torch.int32, device=DEV)
        at += c
    q = torch.randn((sum(rows), hq, d), generator=g, device=DEV).to(torch.bfloat16)
    offsets = torch.tensor([0] + rows, device=DEV).cumsum(0).to(torch.int32)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    return lambda: cat.cat_mx_attention(q, cache, table, length, d ** -0.5, offsets=offsets)


CALLS = {"decode": ([16384] * 16, [1] * 16, 64, 8), "prompts": ([2000, 1500], [2000, 700], 8, 2),
         "parts": ([60000], [70], 8, 1), "mixed": ([2000] + [9000] * 20, [700] + [1] * 20, 32, 8)}


# (at their start decode's CTAs ask for 85 MB at once; with wider heads or more rows copies may have time enough, and none is waited for)
@pytest.mark.parametrize("kind,d", [("decode", 64), ("decode", 128)] + [(k, d) for k in ("prompts", "parts", "mixed") for d in (64, 128, 256)])
def test_bounded_wait_gives_up_then_library_recovers(kind, d):
    run = call(*CALLS[kind], d)
    want = run()
    assert bool(torch.isfinite(want).all())
    assert cat.cat_device_status()[0] == 0
    try:
        cat.cat_set_wait_limit_ns(1)
        run()
        st, word = cat.cat_device_status()
    finally:
        cat.cat_set_wait_limit_ns(0)
    assert st == CAT_ERR_TIMEOUT and word & 1 and word & 1 << 15 and word >> 16, hex(word)
    for _ in range(2):
        assert torch.equal(run(), want)
    assert cat.cat_device_status()[0] == 0


def test_a_limit_that_nothing_reaches():
    """(A tenth of a second: waits look at the clock, and none gives up.)"""
    run = call(*CALLS["mixed"], 128)
    want = run()
    try:
        cat.cat_set_wait_limit_ns(100_000_000)
        got = [run() for _ in range(3)]
        st, word = cat.cat_device_status()
    finally:
        cat.cat_set_wait_limit_ns(0)
    assert st == 0, hex(word)
    assert all(torch.equal(g, want) for g in got)
