"""What the tolerance of tests/test_layer_norm_far_gpu.py tells from what is right, on the CPU: mistakes planted in the values that it is held to."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import delta as R

_spec = importlib.util.spec_from_file_location("far", os.path.join(os.path.dirname(__file__), "test_layer_norm_far_gpu.py"))
far_gpu = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(far_gpu)
f = np.float32


@pytest.mark.parametrize("half", [2.0 ** -24, 2.0 ** -8])
@pytest.mark.parametrize("rows,D,far,spread", far_gpu.FAR)
def test_the_tolerance_tells_other_rows(rng, rows, D, far, spread, half):
    X = (far + spread * rng.normal(size=(rows, D))).astype(f)
    x = X.astype(np.float64)
    c = x - x.mean(-1, keepdims=True)
    v, m = R.layer_norm_fwd(c, eps=0.0)
    n, tol = v["N"], far_gpu.far_tolerance(m["N"], v["N"], c, D, far, half)
    wrong = lambda y: (np.abs(y - n) > tol).mean()  # noqa: E731
    assert wrong(0 * n) > 0.9 and wrong(-n) > 0.9 and wrong(3 * n) > 0.9 and wrong(1.05 * n) > 0.9
    # in fp32: the mean first, then the squares of what is left, and what the mean was off by
    mean = X.sum(-1, keepdims=True, dtype=f) / f(D)
    y = X - mean
    left = y.sum(-1, keepdims=True, dtype=f) / f(D)
    var = (y * y).sum(-1, keepdims=True, dtype=f) / f(D) - left * left
    assert wrong(((y - left) / np.sqrt(var)).astype(np.float64)) == 0
    # and as the mean of squares less the squared mean
    var = np.abs((X * X).sum(-1, keepdims=True, dtype=f) / f(D) - mean * mean) + f(1e-30)
    assert wrong(((X - mean) / np.sqrt(var)).astype(np.float64)) > 0.5
    # the gradient
    dN = rng.normal(size=(rows, D))
    g, gm = R.layer_norm_bwd(c, dN, None, None, 0.0)
    gt = far_gpu.far_tolerance(gm["dX"], g["dX"], c, D, far, half)
    plain = dN / np.sqrt((c ** 2).mean(-1, keepdims=True))
    for y in (0 * g["dX"], -g["dX"], 1.05 * g["dX"], plain + 3 * (plain - g["dX"])):
        assert (np.abs(y - g["dX"]) > gt).mean() > 0.5
