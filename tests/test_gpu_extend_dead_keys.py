"""Scores of minus infinity in attention of new tokens: such a key has weight 0 and counts for nothing, as one that is not
seen, whatever its V; a row that has no other key is 0 / 0.  Bound: that of tests/test_gpu_extend.py, over the other keys."""
import numpy as np
import pytest
import torch

from tests.helpers import f64
from tests.test_gpu_extend import BF, F32, NAN, U, Run

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype, out_dtype", [(BF, BF), (BF, F32), (F32, F32)], ids=str)
@pytest.mark.parametrize("value", [0.5, INF, NAN])
@pytest.mark.parametrize("start, n, dead", [(64, 1, [64]), (300, 2, range(64, 128)), (0, 200, range(0, 130, 3)), (3000, 5, range(40, 2900)), (500, 300, [3, 500, 799])])
@pytest.mark.parametrize("d", [64, 128])
def test_a_score_of_minus_infinity_has_no_weight(start, n, dead, value, d, dtype, out_dtype):
    run = Run([0], 2, d, 4, 28, [(start, n)], dtype=dtype, seed=23)
    q, k, v = run.q[0], run.k[0], run.v[0]
    q[:, :, 0] = q[:, :, 0].abs() + 1
    live = np.ones(start + n, dtype=bool)
    live[list(dead)] = False
    # the definition, over the keys that have a weight
    h, w = torch.finfo(out_dtype).eps / 2, 2.0 ** -8 if out_dtype == BF else 0.0
    j = np.arange(start + n)[live]
    on = j[None] <= start + np.arange(n)[:, None]
    qq, kk, vv = f64(q), f64(k)[live, 0], f64(v)[live, 0]
    want, tol, empty = np.zeros((n, 2, d)), np.zeros((n, 2, d)), ~on.any(1)
    for x in range(2):
        s = np.where(on, qq[:, x] @ kk.T / np.sqrt(d), -np.inf)
        p = np.exp(s - np.where(empty, 0, s.max(1))[:, None])
        p /= np.where(empty, 1, p.sum(1))[:, None]
        want[:, x] = p @ vv
        size = np.where(on, np.abs(qq[:, x]) @ np.abs(kk).T, 0).max(1)[:, None] / np.sqrt(d)
        tol[:, x] = h * np.abs(want[:, x]) + (w + 2 * (d + 3) * U * size + (start + n + 20) * U) * (p @ np.abs(vv))
    k[~live, :, 0] = -INF
    v[~live, :, 3] = value
    run.fill()
    got = f64(run.extend(out_dtype).cpu())
    assert np.isnan(got[empty]).all()  # 0 / 0
    err = np.abs(got - want)[~empty]
    assert np.isfinite(err).all() and (err <= tol[~empty]).all(), float((err / tol[~empty]).max())
