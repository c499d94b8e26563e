"""Packed fp32 rows into the 8-bit caches, bit for bit against the oracle: one chunk of positions a workgroup, two
(sequences of one token at most, and many loosely bounded ones), K and V as slices of one tensor."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2608_06849_amd import aoh_kv_append_q8_varlen, aoh_kv_read_q8
from tests.test_gpu_q8_cache import DEV, Caches, int32, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["mixed", "tokens", "many"])
def test_packed_fp32_rows(kind, d, fmt):
    labels, n_sink, window = [0, 1, 0], 4, 28
    r = np.random.default_rng(d)
    counts, starts, bound = {"mixed": ([0, 1, 16, 70, 33], [9, 15, 0, 5, 100], 70),
                             "tokens": ([1, 0, 1, 1, 1], [9, 3, 0, 15, 31], 1),
                             "many": (r.integers(0, 50, 200).tolist(), r.integers(0, 60, 200).tolist(), 1 << 20)}[kind]
    b, h, top = len(counts), len(labels), max(counts)
    c = Caches(fmt, labels, d, b, 12, n_sink, window, 140)
    kv = rows((sum(counts), 2 * h, d), 140, f"q8-packed32-{kind}", torch.float32) * 1.0009765625  # more bits than bf16
    k, v = kv[:, :h], kv[:, h:]
    cu = np.concatenate([[0], np.cumsum(counts)])
    aoh_kv_append_q8_varlen(k, v, int32(cu.tolist()), bound, labels, int32(starts), c.full, c.ring, n_sink, window)
    kd, vd = (torch.zeros((b, top, h, d), dtype=torch.float32, device=DEV) for _ in range(2))
    for i, n in enumerate(counts):
        kd[i, :n], vd[i, :n] = k[cu[i]:cu[i + 1]], v[cu[i]:cu[i + 1]]
    c.append(kd, vd, starts, counts)
    c.check(kind)
    out = [torch.zeros_like(kd) for _ in range(2)]
    lens = [s + n for s, n in zip(starts, counts)]
    aoh_kv_read_q8(c.full, c.ring, labels, int32(starts), int32(lens), n_sink, window, *out)
    for o, x in zip(out, (kd, vd)):
        want = q8.stored(x.double().cpu().numpy(), fmt)
        for i, n in enumerate(counts):
            p = starts[i] + np.arange(n)
            want[i, :n, 1][(p >= n_sink) & (p < lens[i] - window)] = 0  # not kept by the ring: left as it was
        assert np.array_equal(o.double().cpu().numpy(), want)
