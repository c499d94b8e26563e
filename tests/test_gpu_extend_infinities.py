"""Values of V that are not finite, in attention of new tokens: by the formula a visible infinity has a positive weight and
stays what it is, however small the weight and whatever other sequences hold; both signs, or a NaN, make a NaN.  The rows'
other values keep their bits."""
import numpy as np
import pytest
import torch

from tests.helpers import bits
from tests.test_gpu_extend import BF, F32, NAN, Run

pytestmark = pytest.mark.gpu
INF = float("inf")
# rows and outputs of the three paths
TYPES = [(BF, BF), (BF, F32), (F32, F32)]


@pytest.mark.parametrize("dtype, out_dtype", TYPES, ids=str)
@pytest.mark.parametrize("n, gs", [(3, 2), (5, 7), (40, 4), (200, 2), (300, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_visible_infinity_stays_one(n, gs, d, dtype, out_dtype):
    """Sinks (seen by every row) and a new token, in dimensions of their own."""
    def make():
        return Run([0, 1], gs, d, 4, 24, [(100, n)], dtype=dtype, seed=20)
    want = make().extend(out_dtype).cpu()
    run, at = make(), n // 2
    v = run.v[0]
    v[2, :, 3] = INF
    v[2, :, 7], v[3, :, 7] = INF, -INF
    v[2, :, 9] = NAN
    v[100 + at, :, 5] = -INF
    run.fill()
    got = run.extend(out_dtype).cpu()
    want[:, :, 3] = INF
    want[:, :, 7] = want[:, :, 9] = NAN
    want[at:, :gs, 5] = -INF  # retrieval heads
    want[at:at + 24, gs:, 5] = -INF  # the window of streaming ones
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert np.array_equal(bits(got[~nan]), bits(want[~nan]))


@pytest.mark.parametrize("dtype, out_dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_an_infinity_does_not_depend_on_other_sequences(d, dtype, out_dtype):
    """So many sequences that a workgroup takes several of them; one in seven has a NaN that its first query does not see
    (which sends the workgroup through its tiles again), or a page that is not mapped."""
    def make():
        run = Run([0, 1], 2, d, 4, 28, [(40 + i % 30, 2) for i in range(600)], dtype=dtype, seed=21)
        for v in run.v:
            v[1, :, 3], v[2, :, 4] = INF, -INF
        return run
    run = make()
    run.fill()
    want = run.extend(out_dtype)
    assert (want[:, :, 3] == INF).all() and (want[:, :, 4] == -INF).all()
    other = make()
    for i in range(0, 600, 7):
        other.v[i][-1, :, 11] = NAN  # the second new token
    other.fill()
    for i in range(3, 600, 7):
        other.table[i, 1] = -1
    got = other.extend(out_dtype)
    same = torch.ones(600, dtype=torch.bool)
    same[0::7] = same[3::7] = False
    a, b = (x.unflatten(0, (600, 2)).cpu() for x in (got, want))
    assert np.array_equal(bits(a[same]), bits(b[same]))
    assert np.array_equal(bits(a[0::7, 0]), bits(b[0::7, 0])) and torch.isnan(a[0::7, 1, :, 11]).all()
    keep = torch.arange(d) != 11
    assert np.array_equal(bits(a[0::7, 1][..., keep]), bits(b[0::7, 1][..., keep]))
    assert np.array_equal(bits(a[3::7, :, 2:]), bits(b[3::7, :, 2:]))  # the ring
    assert (a[..., 3] == INF).all() and (a[..., 4] == -INF).all()


@pytest.mark.parametrize("dtype, out_dtype", TYPES, ids=str)
@pytest.mark.parametrize("start, n", [(0, 70), (200, 1), (200, 300), (3000, 3)])
@pytest.mark.parametrize("d", [64, 128])
def test_an_infinity_with_a_weight_below_the_types_range(start, n, d, dtype, out_dtype):
    """The first 70 keys score some hundreds below the others: their weights are 0 in fp32, but not by the formula."""
    def make():
        run = Run([0], 2, d, 4, 28, [(start, n)], dtype=dtype, seed=22)
        run.q[0][:, :, 0] = 32
        run.k[0][:, :, 0] = 0
        run.k[0][:69, :, 0] = -150
        return run
    run = make()
    run.fill()
    want = run.extend(out_dtype).cpu()
    run = make()
    run.v[0][0, :, 3], run.v[0][68, :, 4] = INF, -INF
    run.fill()
    got = run.extend(out_dtype).cpu()
    want[:, :, 3] = INF
    want[max(0, 68 - start):, :, 4] = -INF
    assert np.array_equal(bits(got), bits(want))
