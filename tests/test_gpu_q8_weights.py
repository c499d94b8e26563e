"""Decode over the 8-bit caches keeps every weight whole whatever the type of the output: a bf16 output is off by its own
rounding and by fp32's errors only.

Bound of an output element, with A = sum_j w_j |v_j| (w the exact weights), T keys:
  ds = (D + 4) 2^-24 max_j sum_d |q_d k_jd| / sqrt(D): the scores' error (D products and three multiplications in fp32),
    so a factor exp(2 ds) of a weight at most, and 2^-21 for the exponentials;
  (3 T + 528) 2^-24 for the numerator's sum (three terms a weight, at most 512 partials and 16 more) and
    (T + 528) 2^-24 for the denominator's;
  the output's rounding: torch.finfo(t).eps / 2 of the value.
Weights rounded to bf16 would add 2^-8 A: with values of both signs that is far more than all of these.
"""
import numpy as np
import pytest
import torch

from oracle import attention, q8
from paper_2608_06849_amd import aoh_kv_append_q8
from tests.helpers import f64
from tests.test_gpu_q8_decode import Run

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def check(run, got):
    lens = run.lens.tolist()
    args = (lens, run.labels, run.n_sink, run.window)
    q, top = f64(run.q), max(lens)
    want = attention.decode(q, run.ks, run.vs, *args)
    spread = attention.decode(q, run.ks, np.abs(run.vs), *args)
    big = np.abs(q).reshape(len(lens), len(run.labels), -1, run.d)
    s = np.einsum("bhgd,bthd->bhgt", big, np.abs(run.ks[:, :top])).max(-1) / np.sqrt(run.d)
    ds = (run.d + 4) * 2.0 ** -24 * s.reshape(len(lens), -1, 1)
    exact = (np.expm1(2 * ds) + 2.0 ** -21 + (4 * top + 2 * 528) * 2.0 ** -24) * spread
    bound = exact + torch.finfo(got.dtype).eps / 2 * (np.abs(want) + exact)
    err = np.abs(f64(got) - want)
    assert (err <= bound).all(), f"{(err / bound).max():.2f} of the bound, {(err > bound).sum()} elements"


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
@pytest.mark.parametrize("out", [BF, torch.float32])
@pytest.mark.parametrize("hq,labels,d,lens", [
    (8, [0, 1], 128, [700, 33, 64, 2]),         # work-space pass
    (8, [0, 1], 64, [700, 33, 64, 2]),
    (14, [0, 1], 128, [100, 37] * 40),          # pass of many items
    (16, [1, 0], 64, [100, 37] * 40),
])
def test_no_weight_is_rounded(hq, labels, d, lens, out, fmt):
    run = Run(hq, labels, d, 4, 300, lens, fmt, 110 + d)
    check(run, run.decode(out))


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_values_that_nearly_cancel(fmt):
    # V of odd positions is minus that of the even ones before: what is left is the difference of two weights
    run = Run(6, [0], 128, 0, 1, [400], fmt, 120, kscale=0.02)
    run.v[:, 1::2] = -run.v[:, 0::2]
    aoh_kv_append_q8(run.k.to("cuda"), run.v.to("cuda"), [0], None, run.full, None, 0, 1)
    run.vs = q8.stored(run.v.double().numpy(), fmt)
    check(run, run.decode())
