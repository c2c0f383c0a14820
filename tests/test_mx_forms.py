"""The form that the estimate takes for a product: its accumulators are those that the launch has."""
import pytest

from fake_runtime import FakeRuntime

A = 0x10 << 40          # an address that holds nothing


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return FakeRuntime(tmp_path_factory.mktemp("fake_forms"))


@pytest.mark.parametrize("n,d,d_out,tile", [
    # pairs of 176 and 192 tokens, which have two accumulators: a tile does not wait for the one before to be read
    (4674, 1440, 2176, 192), (1531, 1504, 6784, 192), (650, 2400, 8128, 176), (5874, 1568, 1696, 192),
    # the same tiles where K is short and the outputs' way out counts
    (3634, 352, 2848, 192), (1101, 800, 12384, 192), (2889, 288, 3360, 192),
    # one accumulator
    (8192, 8192, 28672, 256), (2048, 4096, 6144, 240),
])
def test_pairs_of_wide_tiles(fake, n, d, d_out, tile):
    launch, = fake.call("cat_mx_linear", A, A, A, A, n, d, d_out, 1, A, None)
    assert "mx_gemm_kernel<2" in launch.kernel and launch.cluster == 2
    assert fake.box_rows() == [128, tile // 2, 128, tile]
