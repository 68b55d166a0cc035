"""GELU of infinities in the oracle: the limits of z Phi(z)."""
import numpy as np

import oracle
from paper_2411_00288_amd import workloads as wl


def test_gelu_has_its_limits_at_infinities():
    z = np.array([np.inf, -np.inf, np.nan, 1.0, -1.0, 60000.0, -60000.0, 0.0], dtype=np.float32).reshape(1, 2, 4, 1)
    for dtype in (wl.F16, wl.BF16):
        L = wl.Layer("inf", N=1, H=2, W=4, cin=4, cout=1, kh=1, kw=1, dtype=dtype, act=wl.ACT_GELU, mask="top2", seed=1)
        d = wl.make_inputs(L)
        y = oracle.conv2d(d["x"], np.zeros_like(d["W"]), d["M"], cin=4, kh=1, kw=1, dtype=dtype, residual=wl.to_bits(z, dtype), act=wl.ACT_GELU).reshape(-1)
        assert y[0] == np.inf and y[1] == 0.0 and np.isnan(y[2]) and y[7] == 0.0
        assert abs(y[3] - 0.8413447461) < 1e-9 and abs(y[4] + 0.1586552539) < 1e-9
        assert y[5] > 59000 and abs(y[6]) < 1e-12
