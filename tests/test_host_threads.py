"""Calls that are the first CUDA work of their thread, on a runtime without a device: tensor maps are encoded by the
driver, which refuses a thread without a context, and a launch, which would give it one, comes behind them."""
import threading

import pytest

from fake_runtime import FakeRuntime

P = 0x10 << 40          # an address that holds nothing


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    f = FakeRuntime(tmp_path_factory.mktemp("fake_threads"))
    f.lib.fake_want_context(1)
    yield f
    f.lib.fake_want_context(0)


CALLS = {
    "covariance": ("cat_calib_cov", P, 1, 512, 1024, 128, P, 0, None),
    "transform": ("cat_transform_quantize_act", P, 1, 400, 1024, 128, P, P, P, None),
    "weight streaming": ("cat_w4a4_linear", P, P, P, P, 8, 1024, 640, P, None, None),
    "tiles": ("cat_w4a4_linear", P, P, P, P, 300, 1024, 640, P, None, None),
    "byte codes": ("cat_w4a4_linear_e8", P, P, P, P, 300, 1024, 640, P, None, None),
    "digit planes": ("cat_linear_dp", P, 4, 0, P, None, P, 4, P, None, 200, 1024, 640, P, None, None),
    "microscaled": ("cat_mx_linear", P, P, P, P, 40, 1024, 640, 0, P, None),
    "experts": ("cat_mx_linear_grouped", P, P, P, P, P, 2, 40, 1024, 320, 0, P, None),
}


@pytest.mark.parametrize("name", CALLS)
def test_first_cuda_work_of_a_thread(fake, name):
    status = []
    fake.lib.fake_reset()

    def work():
        fake.lib.fake_set_device(3)
        status.append(getattr(fake.lib, CALLS[name][0])(*CALLS[name][1:]))
        status.append(fake.lib.cat_last_error())
    thread = threading.Thread(target=work)
    thread.start()
    thread.join()
    assert status == [0, b""]
    assert fake.lib.fake_boxes() >= 1 and fake.lib.fake_field(0, 0) == 3      # on the thread's device
