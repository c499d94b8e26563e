"""The oracle of the 8-bit caches against the number formats themselves: torch's e4m3 type, exact arithmetic on codes,
the documented error bounds."""
import numpy as np
import pytest
import torch

from oracle import q8


def test_e4m3_codes_are_the_ocp_ones():
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q8.code_values(q8.E4M3), want, equal_nan=True)


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_codes_are_the_nearest_and_ties_go_to_even(fmt):
    table = q8.code_values(fmt)
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-140, 120, (200, 1)))
    x[:50, :8] = 0.0
    grid = np.sort(np.unique(table[np.isfinite(table)]))
    x[50:100] = rng.choice((grid[1:] + grid[:-1]) / 2, (50, 64))  # midpoints, scaled
    x[50:100, 0] = grid.max()
    codes, scales = q8.quantise(x, fmt)
    y = x * np.exp2(127.0 - scales.astype(np.float64))[:, None]
    got = table[codes]
    best = np.abs(y[..., None] - grid).min(-1)
    assert np.array_equal(np.abs(y - got), best)
    tie = (np.abs(y[..., None] - grid) == best[..., None]).sum(-1) > 1
    assert tie[50:100].mean() > 0.5 and np.all(codes[tie] % 2 == 0)


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_scales_are_least_and_errors_bounded(fmt):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((500, 128)) * np.exp2(rng.integers(-135, 124, (500, 1)))
    for i, m in enumerate((1.0, 127.0, 127.0625, 128.0, 448.0, 449.0, 512.0)):
        x[i] = 0.5
        x[i, 7] = -m
    _, scales = q8.quantise(x, fmt)
    e, amax = scales.astype(int) - 127, np.abs(x).max(-1)
    fits = lambda n: amax <= q8.largest(fmt) * np.exp2(n.astype(float))  # noqa: E731
    assert fits(e).all() and (e >= -100).all() and not (fits(e - 1) & (e > -100)).any()
    err = np.abs(q8.stored(x, fmt) - x)
    if fmt == q8.I8:
        assert (err <= np.exp2(e - 1.0)[:, None]).all()
    else:
        assert (err <= np.maximum(np.abs(x) / 16, np.exp2(e - 10.0)[:, None])).all()


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_rows_without_a_scale(fmt):
    x = np.ones((5, 64))
    x[1, 3], x[2, 0], x[3, 63], x[4] = np.nan, -np.inf, 2.0 ** 127, 0.0
    codes, scales = q8.quantise(x, fmt)
    assert scales.tolist()[1:] == [255, 255, 255, 27] and not codes[1:].any()
    assert np.isnan(q8.values(codes, scales, fmt)[1:4]).all() and not q8.values(codes, scales, fmt)[4].any()


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_stored_values_are_stored_as_themselves(fmt):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((300, 64)) * np.exp2(rng.integers(-140, 120, (300, 1)))
    # a maximum that rounds down to half of the largest code: the next scale below holds it as well
    x[:40] = rng.standard_normal((40, 64)) * 8
    x[:40, 0] = q8.largest(fmt) / 2 * (1 + 2.0 ** -6)
    once = q8.stored(x, fmt)
    assert np.array_equal(q8.stored(once, fmt), once)


def test_v_layout_round_trip():
    rows = np.arange(2 * 16 * 64).reshape(2, 16, 64)
    unit = q8.v_unit(rows)
    assert unit.shape == (2, 16, 4, 4, 4)
    for r, d in ((0, 0), (5, 9), (15, 63), (7, 30)):
        assert unit[1, d // 4, r // 4, d % 4, r % 4] == rows[1, r, d]
    assert np.array_equal(q8.v_rows(unit), rows)
