"""The transforms in front of the microscaled form: x' = T x and W' = W T^-1 from the library, quantized and multiplied.

The signal-to-quantization-noise ratio of the output is that of the definition in float64 (the same T, x' and W' exact,
quantized by mx_reference).  A code differs only where float32's x' or W' (within about 1e-6) falls on the other side of a tie,
where both neighbours are equally far: 0.01 dB is far more than such values, one in 10^5, can move."""
import numpy as np
import pytest
import torch

import mx_reference as R
import workloads as WL
from test_gpu_mx import cat, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["lowrank_outlier", "swiglu"])
@pytest.mark.parametrize("kind,k", [("identity", 64), ("rht", 128), ("cat", 32), ("cat", 128)])
def test_sqnr_of_a_transformed_layer(kind, k, act):
    cfg = WL.small_config("mx", d_in=1024, d_out=384, n_eval=300, n_calib=512, k=k, seed=31, act=act, outlier_frac=0.01,
                          outlier_scale=100.0)
    L = WL.make_layer(cfg)
    x, W, xc = (dev(t.values, torch.bfloat16 if t.dtype == "bf16" else torch.float32) for t in (L.x_eval, L.W, L.x_calib))
    sigma = cat.cat_calib_cov(xc, k) if kind == "cat" else None
    T, _, _ = cat.cat_quantize_weights(W, k, kind, sigma_x=sigma, n_calib=cfg.n_calib,
                                       rht_signs=L.rht_signs if kind == "rht" else None)
    Tinv = torch.linalg.inv(T.double()).float().contiguous()
    xt, wt = cat.cat_block_transform(x, k, T), cat.cat_block_transform(W, k, Tinv, transpose=True)
    y = cat.cat_mx_linear(*cat.cat_mx_quantize(xt), *cat.cat_mx_quantize(wt))
    want = x.float() @ W.float().T
    got = float(cat.cat_sqnr(want.contiguous(), y)[2])

    def blocks(v, m):
        return np.einsum("rbj,bij->rbi", v.reshape(v.shape[0], -1, k), m).reshape(v.shape)
    x64, w64, t64, i64 = (a.double().cpu().numpy() for a in (x, W, T, Tinv))
    xv = R.values(*R.quantize(blocks(x64, t64)))
    wv = R.values(*R.quantize(blocks(w64, i64.transpose(0, 2, 1))))
    y64 = x64 @ w64.T
    exact = 10 * np.log10((y64 ** 2).sum() / ((xv @ wv.T - y64) ** 2).sum())
    assert abs(got - exact) <= 0.01, (got, exact)
    assert cat.cat_device_status()[0] == 0
