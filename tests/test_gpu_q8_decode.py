"""Decode over the 8-bit caches (aoh_decode_q8, aoh_decode_step_q8) against the float64 oracle on the values that the
oracle's own quantisation gives, with bounds that follow from the arithmetic.

Bound of an output element, with A = sum_j w_j |v_j| (w the exact weights), T keys:
  scores: D exact products summed in fp32, and three multiplications after it: off by at most
    ds = (D + 4) 2^-24 max_j sum_d |q_d k_jd| / sqrt(D); so a weight by a factor exp(2 ds) at most (its own score and
    the sum's), plus 2^-21 for the exponentials, whose arguments in log2 units are rounded once more;
  weights: to bf16 for a bf16 output, half a step of which is 2^-8 of the weight (torch.finfo(torch.bfloat16).eps / 2);
    for an fp32 output as three bf16 numbers of 8 significant bits each, which hold fp32's 24;
  sums over T keys in fp32, joined over at most 512 partials: (T + 512 + 16) 2^-24 of the absolute sum, for numerator
    and denominator (the three parts of a weight are three terms of the numerator);
  the output's rounding: 2^-8 of the value (bf16) or 2^-24 (fp32).
"""
import numpy as np
import pytest
import torch

import synth
from oracle import attention, q8
from paper_2608_06849_amd import (AohError, PagedCacheQ8, RingCacheQ8, aoh_decode_q8, aoh_decode_q8_workspace_bytes,
                                  aoh_decode_step_q8, aoh_kv_append_q8, aoh_kv_append_q8_varlen, aoh_kv_read_q8,
                                  aoh_prefill_varlen)
from tests.helpers import bits, f64
from tests.test_gpu_q8_cache import DTYPES, int32, raw

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


class Run:
    """Sequences of these lengths in 8-bit caches whose other bytes are NaN codes and infinite scales."""

    def __init__(self, hq, labels, d, n_sink, window, lens, fmt, seed, extra_pages=1, kscale=0.5, tail=0):
        b, h = len(lens), len(labels)
        self.hq, self.labels, self.d, self.n_sink, self.window, self.fmt = hq, labels, d, n_sink, window, fmt
        top = max(max(lens), 1) + tail
        # a cheap source of rows: a block of random ones, shifted for each sequence and head
        base = synth.gaussian((top + 97 * min(b * h, 53), d), seed, "q8-base").astype(np.float32)
        self.k, self.v = (np.empty((b, top, h, d), dtype=np.float32) for _ in range(2))
        for i in range(b):
            for g in range(h):
                o = 97 * ((i * h + g) % 53)
                self.k[i, :, g] = base[o:o + top] * kscale
                self.v[i, :, g] = np.roll(base[o:o + top], 1 + g + i, axis=1)
        self.k, self.v = (torch.from_numpy(x).to(BF) for x in (self.k, self.v))
        self.q = torch.from_numpy(synth.gaussian((b, hq, d), seed, "q8-q").astype(np.float32)).to(BF).to(DEV)
        pages = (top + 15) // 16 + extra_pages
        table = synth.page_permutation(b * pages, seed, "q8-pages").reshape(b, pages).astype(np.int32)
        for i, n in enumerate(lens):  # entries past the end are unmapped
            table[i, (n + tail + 15) // 16:] = (-1, 1 << 30)[i % 2]
        n_ret = labels.count(0)
        dt = DTYPES[fmt]
        self.full = PagedCacheQ8.allocate(b * pages, n_ret, d, dt, torch.from_numpy(table)) if n_ret else None
        self.ring = RingCacheQ8.allocate(b, h - n_ret, n_sink, window, d, dt) if n_ret < h else None
        for c in (self.full, self.ring):
            if c:
                c.k.view(torch.uint8).fill_(0x7F)
                c.v.view(torch.uint8).fill_(0xFF)
                c.scales.fill_(255)
        cu = np.concatenate([[0], np.cumsum(lens)])
        self.lens = int32(lens)
        if cu[-1]:
            k, v = (torch.cat([x[i, :n] for i, n in enumerate(lens)]).to(DEV) for x in (self.k, self.v))
            aoh_kv_append_q8_varlen(k, v, int32(cu.tolist()), max(lens), labels, None, self.full, self.ring, n_sink, window)
        self.ks, self.vs = (q8.stored(x.double().numpy(), fmt) for x in (self.k, self.v))

    @property
    def caches(self):
        return [raw(t) for c in (self.full, self.ring) if c for t in (c.k, c.v, c.scales)]

    def decode(self, out=BF, **kw):
        o = torch.full(self.q.shape, 7.0, dtype=out, device=DEV)
        return aoh_decode_q8(self.q, self.full, self.ring, self.labels, self.lens, self.n_sink, self.window, out=o, **kw)

    def check(self, got, lens=None, what=""):
        lens = self.lens.tolist() if lens is None else lens
        on = [i for i, n in enumerate(lens) if n > 0]
        g = f64(got)
        assert not g[[i for i, n in enumerate(lens) if n <= 0]].any(), f"{what}: empty sequences"
        if not on:
            return
        args = ([lens[i] for i in on], self.labels, self.n_sink, self.window)
        q = f64(self.q)[on]
        want = attention.decode(q, self.ks[on], self.vs[on], *args)
        spread = attention.decode(q, self.ks[on], np.abs(self.vs[on]), *args)
        top = max(lens)
        big = np.abs(q).reshape(len(on), len(self.labels), -1, self.d)
        s = np.einsum("bhgd,bthd->bhgt", big, np.abs(self.ks[on][:, :top])).max(-1) / np.sqrt(self.d)
        ds = (self.d + 4) * 2.0 ** -24 * s.reshape(len(on), -1, 1)
        weight, parts = (2.0 ** -8, 1) if got.dtype == BF else (0.0, 3)
        rel = np.expm1(2 * ds) + 2.0 ** -21 + weight + ((1 + parts) * top + 2 * 528) * 2.0 ** -24
        step = 2.0 ** -8 if got.dtype == BF else 2.0 ** -24
        err = np.abs(g[on] - want)
        bound = rel * spread + step * (np.abs(want) + rel * spread)
        assert (err <= bound).all(), f"{what}: {(err / bound).max():.2f} of the bound"


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 0, 500, 1027, 300]
GROUPS = [  # hq, labels, d, n_sink, window
    (1, [0], 128, 0, 1),
    (1, [1], 64, 0, 1),
    (4, [0, 1, 0, 1], 64, 4, 29),
    (14, [0, 1], 128, 16, 112),
    (15, [1, 0, 0, 1, 0], 128, 0, 77),
    (32, [0, 1], 64, 3, 30),
    (8, [0, 0], 128, 64, 1024),
    (9, [1, 1, 1], 128, 128, 256),
]


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
@pytest.mark.parametrize("out", [BF, torch.float32])
@pytest.mark.parametrize("hq,labels,d,n_sink,window", GROUPS)
def test_decode_ragged_lengths(hq, labels, d, n_sink, window, out, fmt):
    run = Run(hq, labels, d, n_sink, window, LENS, fmt, 31 + hq)
    before = run.caches
    got = run.decode(out)
    run.check(got, what="decode")
    assert all(np.array_equal(a, b) for a, b in zip(before, run.caches))
    assert torch.equal(got, run.decode(out)), "a second run gives other bits"


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
@pytest.mark.parametrize("batch,labels,hq", [(1, [0, 1], 8), (64, [0, 1, 0], 12), (65, [1, 0], 2), (130, [0, 1, 1, 0], 16)])
def test_batches_of_both_split_passes(batch, labels, hq, fmt):
    r = np.random.default_rng(batch)
    run = Run(hq, labels, 64, 4, 60, r.integers(0, 200, batch).tolist(), fmt, batch)
    run.check(run.decode(torch.float32), what="fp32 out")
    run.check(run.decode(), what="bf16 out")


@pytest.mark.parametrize("batch,full", [(200, [70, 71, 127, 193, 199]), (129, [128]), (128, [0]), (300, []), (1024, [63, 64, 1023])])
def test_batches_with_long_empty_stretches(batch, full):
    lens = [0] * batch
    for i in full:
        lens[i] = 5 + 37 * (i % 7)
    run = Run(4, [0, 1], 64, 4, 60, lens, q8.I8, 7, tail=1)
    run.check(run.decode(torch.float32))
    step_and_two_calls(run, BF)


def test_more_sequences_than_a_launch_takes():
    r = np.random.default_rng(5)
    run = Run(2, [0, 1], 64, 4, 28, r.integers(0, 40, 2100).tolist(), q8.I8, 6, tail=1)
    run.check(run.decode())
    # with the step's token, which the last part of the batch (fewer than 64 sequences) stores too
    step_and_two_calls(run, torch.float32)


@pytest.mark.parametrize("d,length", [(128, 70001), (64, 100000)])
def test_one_long_sequence_is_split(d, length):
    run = Run(6, [0, 1], d, 64, 1000, [length], q8.E4M3, 9)
    run.check(run.decode(torch.float32))


@pytest.mark.parametrize("lens", [[1, 3000], [2500] + [1] * 20, [0, 17, 0, 1, 1900, 16], [40] * 30])
@pytest.mark.parametrize("hq,labels,d", [(8, [0] * 8, 64), (6, [1, 0, 1], 128), (2, [1, 1], 128)])
def test_short_and_long_sequences_together(hq, labels, d, lens):
    run = Run(hq, labels, d, 4, 1500, lens, q8.E4M3, 12, tail=1)
    run.check(run.decode(torch.float32))
    step_and_two_calls(run, BF)


def test_lengths_beyond_the_table_are_clamped():
    run = Run(2, [0], 64, 0, 1, [64, 32], q8.I8, 10, extra_pages=0)
    full = PagedCacheQ8(run.full.k, run.full.v, run.full.scales, run.full.block_table[:, :2].contiguous())
    got = aoh_decode_q8(run.q, full, None, [0], int32([64, 1 << 30]), 0, 1)
    run.check(got, [32, 32])


def step_and_two_calls(run, out=BF):
    """One fused step, checked against append + decode on a copy of the caches; leaves the token in the run."""
    start = run.lens.clone()
    copy = [type(c)(c.k.clone(), c.v.clone(), c.scales.clone(), c.block_table if c is run.full else c.capacity)
            if c else None for c in (run.full, run.ring)]
    at = start.long().cpu()
    i = torch.arange(len(at))
    kn, vn = (x[i, at].to(DEV) for x in (run.k, run.v))
    run.lens = start + 1
    got = aoh_decode_step_q8(run.q, kn, vn, run.full, run.ring, run.labels, run.lens, run.n_sink, run.window,
                             out=torch.empty(run.q.shape, dtype=out, device=DEV))
    aoh_kv_append_q8(kn.unsqueeze(1), vn.unsqueeze(1), run.labels, start, *copy, run.n_sink, run.window)
    want = aoh_decode_q8(run.q, *copy, run.labels, run.lens, run.n_sink, run.window,
                         out=torch.empty(run.q.shape, dtype=out, device=DEV))
    assert np.array_equal(bits(got), bits(want)), "the step's output"
    for a, b in zip(copy, (run.full, run.ring)):
        for x, y in zip((a.k, a.v, a.scales) if a else (), (b.k, b.v, b.scales) if b else ()):
            assert np.array_equal(raw(x), raw(y)), "the step's caches"
    run.check(got)


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
@pytest.mark.parametrize("hq,labels,d,n_sink,window", GROUPS)
@pytest.mark.parametrize("batch", [18, 70])
def test_step_equals_append_then_decode(batch, hq, labels, d, n_sink, window, fmt):
    lens = [0, 15, 16, 31, 32, 33, 63, 64, 65, 100, 127, 128, 3, 7, 200, 48, 47, 17]
    run = Run(hq, labels, d, n_sink, window, (lens * 4)[:batch], fmt, 50 + hq, extra_pages=1, tail=2)
    for _ in range(2):
        step_and_two_calls(run)


def test_step_at_places_without_a_page():
    # an unmapped page gets no token; an empty place of the batch gets none either, and 0
    run = Run(4, [0, 1], 64, 4, 28, [31, 32, 20], q8.E4M3, 12, tail=1)
    table = run.full.block_table.clone()
    table[1, 2] = -1
    full = PagedCacheQ8(run.full.k, run.full.v, run.full.scales, table)
    before = [raw(t) for t in (full.k, full.v, full.scales, run.ring.k, run.ring.v, run.ring.scales)]
    kn = torch.ones((3, 2, 64), dtype=BF, device=DEV)
    got = aoh_decode_step_q8(run.q, kn, kn, full, run.ring, [0, 1], int32([32, 33, 0]), 4, 28)
    after = [raw(t) for t in (full.k, full.v, full.scales, run.ring.k, run.ring.v, run.ring.scales)]
    page = int(table[0, 1])
    for x, y in zip(before[:3], after[:3]):
        x, y = np.delete(x, page, 0), np.delete(y, page, 0)
        assert np.array_equal(x, y)
    for x, y in zip(before[3:], after[3:]):
        assert np.array_equal(x[2], y[2]) and not np.array_equal(x[:2], y[:2])
    assert not got[2].any() and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_rows_of_nan_reach_their_heads_only(fmt):
    run = Run(4, [0, 1], 128, 4, 60, [100, 100, 100, 100], fmt, 13)
    want = f64(run.decode())
    kv = [run.k[:, 99:100].clone(), run.v[:, 99:100].clone()]
    kv[0][1, 0, 0, 3] = float("nan")    # K of sequence 1, retrieval head
    kv[1][2, 0, 1, 5] = float("inf")    # V of sequence 2, streaming head
    aoh_kv_append_q8(*(x.to(DEV) for x in kv), run.labels, run.lens - 1, run.full, run.ring, 4, 60)
    got = f64(run.decode())
    nan = np.zeros((4, 4), dtype=bool)
    nan[1, :2] = nan[2, 2:] = True
    assert np.isnan(got[nan]).all() and np.array_equal(got[~nan], want[~nan])


def test_large_and_small_magnitudes():
    # scores of some hundreds, V over 200 binades: one weight is 1, the others far below
    run = Run(2, [0], 64, 0, 1, [200], q8.E4M3, 14, kscale=30.0)
    run.check(run.decode(torch.float32))
    v = run.v[:1, :200].float() * torch.exp2(torch.arange(200).float() - 100).view(1, -1, 1, 1)
    run.v[:1, :200] = v.to(BF)
    aoh_kv_append_q8(run.k[:1, :200].to(DEV), run.v[:1, :200].to(DEV), [0], None, run.full, None, 0, 1)
    run.vs = q8.stored(run.v.double().numpy(), q8.E4M3)
    run.check(run.decode(torch.float32))


def test_equal_keys_give_the_mean_and_one_key_its_value():
    for n in (1, 5, 64, 777):
        run = Run(3, [0], 128, 0, 1, [n], q8.I8, 15, kscale=0.0)
        got = f64(run.decode(torch.float32))[0]
        assert np.abs(got - run.vs[0, :n, 0].mean(0)).max() <= (n + 600) * 2.0 ** -23 * np.abs(run.vs).max()
        if n == 1:
            assert np.array_equal(got[2], run.vs[0, 0, 0])


def test_strided_queries_outputs_and_a_side_stream():
    run = Run(8, [0, 1], 64, 4, 60, [90, 33, 150], q8.I8, 16, tail=1)
    want = run.decode()
    wide = torch.zeros((3, 3, 8, 64), dtype=BF, device=DEV)
    wide[:, 0] = run.q
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    # on the given stream, while the current one is another
    aoh_decode_q8(wide[:, 0], run.full, run.ring, run.labels, run.lens, 4, 60, out=wide[:, 2], stream=s)
    s.synchronize()
    assert torch.equal(wide[:, 2], want) and not wide[:, 1].any()


def test_two_graphs_with_eager_work_between():
    # two captured steps that keep a workspace each, replayed in turn with eager steps of other lengths between
    runs = [Run(8, [0, 1, 1, 0], 128, 4, 60, lens, q8.E4M3, 20 + len(lens), tail=1) for lens in ([300, 7], [40] * 70)]
    graphs, outs, wants = [], [], []
    for run in runs:
        at = run.lens.long().cpu()
        i = torch.arange(len(at))
        kn, vn = (x[i, at].to(DEV) for x in (run.k, run.v))
        run.lens = run.lens + 1
        out, ws = torch.zeros_like(run.q), torch.zeros(aoh_decode_q8_workspace_bytes(len(at), 8, 128), dtype=torch.uint8,
                                                       device=DEV)
        args = (run.q, kn, vn, run.full, run.ring, run.labels, run.lens, 4, 60)
        wants.append(aoh_decode_step_q8(*args).clone())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            aoh_decode_step_q8(*args, out=out, workspace=ws)
        graphs.append((g, kn, vn, ws))
        outs.append(out)
    for n in range(4):
        for (g, *_), out, want, run in zip(graphs, outs, wants, runs):
            out.fill_(7.0)
            g.replay()
            run.decode(torch.float32)
            assert torch.equal(out, want), f"replay {n}"
    # the captured call follows the lengths in the tensor
    runs[0].lens.sub_(1)
    graphs[0][0].replay()
    assert not torch.equal(outs[0], wants[0])


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_prompts_then_captured_steps_then_read(fmt):
    """The calls as a serving program makes them: packed prompts attended to and written, steps in one graph, the
    sequence handed on as bf16 values."""
    hq, labels, d, n_sink, window, steps = 8, [1, 0], 128, 16, 112, 5
    lens = [37, 260, 16]
    run = Run(hq, labels, d, n_sink, window, [0, 0, 0], fmt, 60, extra_pages=20)
    run = Run(hq, labels, d, n_sink, window, lens, fmt, 60, tail=steps)
    q = torch.from_numpy(synth.gaussian((sum(lens), hq, d), 61, "q8-prompt").astype(np.float32)).to(BF).to(DEV)
    k, v = (torch.cat([x[i, :n] for i, n in enumerate(lens)]).to(DEV) for x in (run.k, run.v))
    cu = int32([0, 37, 297, 313])
    for c in (run.full, run.ring):
        c.scales.fill_(255)
    prompt = aoh_prefill_varlen(q, k, v, cu, max(lens), labels, n_sink, window)
    aoh_kv_append_q8_varlen(k, v, cu, max(lens), labels, None, run.full, run.ring, n_sink, window)
    assert torch.isfinite(prompt).all()
    kn, vn = torch.zeros((3, 2, d), dtype=BF, device=DEV), torch.zeros((3, 2, d), dtype=BF, device=DEV)
    ws = torch.empty(aoh_decode_q8_workspace_bytes(3, hq, d), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(run.q)
    now = run.lens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        now += 1
        aoh_decode_step_q8(run.q, kn, vn, run.full, run.ring, labels, now, n_sink, window, out=out, workspace=ws)
    now.copy_(run.lens)
    for s in range(steps):
        for i, n in enumerate(lens):
            kn[i], vn[i] = run.k[i, n + s].to(DEV), run.v[i, n + s].to(DEV)
        graph.replay()
        torch.cuda.synchronize()
        run.check(out, [n + s + 1 for n in lens], f"step {s}")
    total = max(lens) + steps
    got = [torch.zeros((3, total, 2, d), dtype=BF, device=DEV) for _ in range(2)]
    aoh_kv_read_q8(run.full, run.ring, labels, None, now, n_sink, window, *got)
    for x, want in zip(got, (run.ks, run.vs)):
        x = f64(x)
        for i, n in enumerate(lens):
            n += steps
            assert np.array_equal(x[i, :n, 1], want[i, :n, 1]) and not x[i, n:].any()
            assert np.array_equal(x[i, max(0, n - window):n, 0], want[i, max(0, n - window):n, 0])


def test_refused_calls_leave_the_output():
    run = Run(4, [0, 1], 64, 4, 28, [10, 20], q8.I8, 70)
    out = torch.full(run.q.shape, 7.0, dtype=BF, device=DEV)
    with pytest.raises(AohError):
        aoh_decode_q8(run.q, run.full, run.ring, [0, 1], run.lens, 4, 29, out=out)
    with pytest.raises(AohError):
        aoh_decode_q8(run.q, run.full, run.ring, [0, 1], run.lens, 4, 28, out=out,
                      workspace=torch.empty(1000, dtype=torch.uint8, device=DEV))
    with pytest.raises(AohError):
        aoh_decode_q8(run.q.float(), run.full, run.ring, [0, 1], run.lens, 4, 28, out=out)
    with pytest.raises(ValueError):
        aoh_decode_q8(run.q, run.full, run.ring, [0, 1], run.lens.long(), 4, 28, out=out)
    with pytest.raises(ValueError):
        aoh_decode_q8(run.q, run.full, run.ring, [0, 1], run.lens[:1], 4, 28, out=out)
    with pytest.raises(ValueError):
        aoh_decode_q8(run.q, run.full, run.ring, [0], run.lens, 4, 28, out=out)
    torch.cuda.synchronize()
    assert (out == 7.0).all()
