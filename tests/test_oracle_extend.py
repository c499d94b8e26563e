"""The oracle of attention behind a cached prefix against the prefill's."""
import numpy as np
import pytest

from oracle import attention, extend

STREAMING, HQ, HKV, D = [0, 1], 4, 2, 8


def rows(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("chunk", [1, 3, 7, 40])
@pytest.mark.parametrize("evict", [False, True])
def test_chunk_after_chunk_is_the_prefill(chunk, evict):
    n, n_sink, window = 40, 3, 6
    q, k, v = rows(1, n, HQ, D), rows(2, n, HKV, D), rows(3, n, HKV, D)
    got = np.concatenate([extend.extend(q[s:s + chunk], k[:s + chunk], v[:s + chunk], s, STREAMING, n_sink, window, evict)[0]
                          for s in range(0, n, chunk)])
    for h in range(HQ):
        g = attention.group_of(h, HQ, HKV)
        want = attention.attend_rows(q[:, h], np.arange(n), k[:, g], v[:, g], STREAMING[g], n_sink, window, chunk if evict else 0)
        assert np.allclose(got[:, h], want, atol=1e-12)


def test_visible_by_hand():
    assert extend.visible(10, [0, 2], True, 1, 3, False).astype(int).tolist() == [
        [1, 0, 0, 0, 0, 0, 0, 0, 1, 1, 1, 0, 0], [1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1, 1, 1]]
    assert extend.visible(10, [0, 2], True, 1, 3, True).astype(int).tolist() == [
        [1, 0, 0, 0, 0, 0, 0, 1, 1, 1, 1, 0, 0], [1, 0, 0, 0, 0, 0, 0, 1, 1, 1, 1, 1, 1]]
    assert extend.visible(2, [1], False, 1, 1, False).astype(int).tolist() == [[1, 1, 1, 1]]


def test_masses_bound_the_output():
    q, k, v = rows(1, 5, HQ, D), rows(2, 12, HKV, D), rows(3, 12, HKV, D)
    out, mass, size = extend.extend(q, k, v, 7, STREAMING, 1, 3, False)
    assert (np.abs(out) <= mass + 1e-15).all() and (size > 0).all()
    assert np.allclose(extend.extend(q, k, v, 7, STREAMING, 1, 3, False, rows=[4, 1])[0], out[[4, 1]])
