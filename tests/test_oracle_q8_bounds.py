"""The error bounds that the C header states for the 8-bit formats, on both sides of the least scale, and what becomes of
values whose scaled form fp32 cannot hold."""
import numpy as np
import pytest
import torch

from oracle import q8


def rows(low, high, n=2000, d=64):
    r = np.random.default_rng(n + d)
    return (r.standard_normal((n, d)) * np.exp2(r.integers(low, high, (n, 1)))).astype(np.float32).astype(np.float64)


def test_int8_error_is_below_a_127th_of_the_maximum_above_the_least_scale():
    x = rows(-85, 120)
    _, scale = q8.quantise(x, q8.I8)
    e = scale.astype(int) - 127
    assert (e > -100).all()
    err, amax = np.abs(q8.stored(x, q8.I8) - x).max(-1), np.abs(x).max(-1)
    assert (err <= np.exp2(e - 1.0)).all() and (np.exp2(e - 1.0) < amax / 127).all()


@pytest.mark.parametrize("fmt,absolute", [(q8.I8, 2.0 ** -101), (q8.E4M3, 2.0 ** -110)])
def test_rows_at_the_least_scale_keep_an_absolute_bound(fmt, absolute):
    x = rows(-126, -107)
    _, scale = q8.quantise(x, fmt)
    assert (scale == 27).all()
    err = np.abs(q8.stored(x, fmt) - x)
    small = np.abs(x) < 2.0 ** -106 if fmt == q8.E4M3 else np.ones_like(x, dtype=bool)
    assert (err[small] <= absolute).all() and (err[~small] <= np.abs(x[~small]) / 16).all()
    gone = np.abs(x).max(-1) < absolute
    assert gone.any() and not q8.stored(x, fmt)[gone].any()
    if fmt == q8.I8:  # the relative bound does not reach here
        assert (err.max(-1) > np.abs(x).max(-1) / 127).any()


@pytest.mark.parametrize("fmt", [q8.I8, q8.E4M3])
def test_values_below_the_normal_range_once_scaled_have_code_zero(fmt):
    x = rows(-20, 100)
    x[:, 1::2] = 2.0 ** np.random.default_rng(5).integers(-149, -20, x[:, 1::2].shape)
    codes, scale = q8.quantise(x, fmt)
    factor = np.exp2(127.0 - scale.astype(np.float64))[:, None]
    exact = x * factor
    low = np.abs(exact) < 2.0 ** -126
    assert low.any() and not (codes[low] & 127).any()
    # everywhere else the product is exact in fp32
    f32 = torch.from_numpy(x).float() * torch.from_numpy(factor).float()
    assert np.array_equal(f32.double().numpy()[~low], exact[~low])
