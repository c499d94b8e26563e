"""Attention of new tokens over the caches and themselves, against the float64 oracle on the logical sequence.

The caches are filled with NaN before the prefix is appended, and rows behind a sequence's end hold NaN, so that whatever
is read without being seen shows.  Two kinds of checks:

counts   K = 0, so that every visible key weighs the same, and V of random zeros and ones: an output times the number of
         visible keys is the number of ones among them, a whole number that any key too many or too few changes in half
         of the dimensions.  Weights are 1 whatever their type, sums of ones are exact: only the division rounds.
values   random rows, within a bound (u = 2^-24, h half a step of the output's dtype, w = 2^-8 where weights are rounded
         to bf16 for a bf16 output, 0 else): a score is off by at most (D + 3) u sum_d |q_d k_d| / sqrt(D) (D fp32 sums of
         exact products; the factor, the difference to the maximum), its weight by twice that (numerator and denominator)
         and 4 u of exp2 and of rescaling; n products are summed in fp32: n u; merging adds 16 u:
         |error| <= h |o| + (w + 2 (D + 3) u size + (n + 20) u) sum_j w_j |v_j|."""
import numpy as np
import pytest
import torch

import synth
from oracle import extend as oracle
from paper_2608_06849_amd import (PagedCache, RingCache, aoh_extend, aoh_extend_varlen, aoh_extend_workspace_bytes, aoh_kv_append,
                                  aoh_prefill, aoh_prefill_chunked)
from tests.helpers import bits, f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
NAN = float("nan")


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(DEV)


class Run:
    """Sequences of (start, new) tokens in caches that hold the first `start` of them; spare pages and block-table
    entries lie around."""

    def __init__(self, labels, gs, d, n_sink, window, seqs, dtype=BF, seed=0, count=False, spare=2):
        self.labels, self.gs, self.d, self.n_sink, self.window, self.seqs, self.dtype = labels, gs, d, n_sink, window, seqs, dtype
        hkv, b = len(labels), len(seqs)
        self.hkv, self.hq, self.b = hkv, hkv * gs, b
        self.starts, self.new = [s for s, _ in seqs], [n for _, n in seqs]
        r = np.random.default_rng(1000 + seed)
        self.q, self.k, self.v = [], [], []
        for s, n in seqs:
            q, k, v = (r.standard_normal((t, h, d), dtype=np.float32) for t, h in ((n, self.hq), (s + n, hkv), (s + n, hkv)))
            if count:
                k, v = k * 0, (v > 0).astype(np.float32)
            self.q.append(torch.from_numpy(q).to(dtype))
            self.k.append(torch.from_numpy(k).to(dtype))
            self.v.append(torch.from_numpy(v).to(dtype))
        self.pages = (max(s + n for s, n in seqs) + 15) // 16 + spare
        perm = synth.page_permutation(b * self.pages + 3, 7 + seed, "pages")
        self.table = torch.from_numpy(perm[:b * self.pages].reshape(b, self.pages).astype(np.int32)).to(DEV)
        for i, (s, n) in enumerate(seqs):
            self.table[i, (s + n + 15) // 16:] = -1
        self.fill()

    def fill(self):
        d, b = self.d, self.b
        self.full = PagedCache.allocate(b * self.pages + 3, self.labels.count(0), d, self.dtype, self.table) if 0 in self.labels else None
        self.ring = RingCache.allocate(b, self.labels.count(1), self.n_sink, self.window, d, self.dtype) if 1 in self.labels else None
        for t in self.tensors():
            t.fill_(NAN)
        for i, s in enumerate(self.starts):
            if s:
                self.append(i, 0, s, self.full, self.ring)

    def append(self, i, lo, hi, full, ring):
        full = full.rows(i, i + 1) if full is not None else None
        ring = RingCache(ring.k[i:i + 1], ring.v[i:i + 1], ring.capacity) if ring is not None else None
        aoh_kv_append(self.k[i][None, lo:hi].to(DEV), self.v[i][None, lo:hi].to(DEV), self.labels, i32([lo]), full, ring, self.n_sink,
                      self.window)

    def tensors(self):
        return [t for c in (self.full, self.ring) if c is not None for t in (c.k, c.v)]

    def packed(self, tail=3):
        """q, k, v [total + tail, H, D], slices of one tensor, with NaN behind the last sequence; cu_seqlens."""
        rows = torch.cat([torch.cat([q, k[s:], v[s:]], 1) for q, k, v, s in zip(self.q, self.k, self.v, self.starts)] +
                         [torch.full((tail, self.hq + 2 * self.hkv, self.d), NAN, dtype=self.dtype)]).to(DEV)
        h = self.hq
        return rows[:, :h], rows[:, h:h + self.hkv], rows[:, h + self.hkv:], i32(np.concatenate([[0], np.cumsum(self.new)]))

    def extend(self, out_dtype=None, evict=False, append=False, **kw):
        """Packed outputs of the sequences, [total, Hq, D]."""
        q, k, v, cu = self.packed()
        out = torch.full(q.shape, 7.0, dtype=out_dtype or self.dtype, device=DEV)
        aoh_extend_varlen(q, k, v, cu, max(self.new), self.labels, i32(self.starts), self.full, self.ring, self.n_sink, self.window,
                          evict=evict, append=append, out=out, **kw)
        assert (out[int(cu[-1]):] == 7).all()
        return out[:int(cu[-1])]

    def check_counts(self, out, evict=False):
        at = 0
        for s, n, v in zip(self.starts, self.new, self.v):
            if n == 0:
                continue
            for g, m in enumerate(self.labels):
                on = torch.from_numpy(oracle.visible(s, np.arange(n), m, self.n_sink, self.window, evict)).double()
                ones, total = on @ v[:, g].double(), on.sum(1, keepdim=True)
                got = out[at:at + n, g * self.gs:(g + 1) * self.gs].cpu().double() * total[:, None]
                off = (got - ones[:, None]).abs().max(-1).values.max(-1).values
                assert off.max() < 0.01, f"start {s}, new {n}, head {g}: rows {(~(off < 0.01)).nonzero().flatten().tolist()[:9]}, {off.max()}"
            at += n

    def check_values(self, out, evict=False, rows=None, skip=()):
        at, worst = 0, 0.0
        h = torch.finfo(out.dtype).eps / 2
        w = 2.0 ** -8 if out.dtype == BF else 0.0
        for i, (s, n) in enumerate(self.seqs):
            if n and i not in skip:
                pick = np.arange(n) if rows is None else np.unique(np.clip(rows, 0, n - 1))
                o, mass, size = oracle.extend(f64(self.q[i]), f64(self.k[i]), f64(self.v[i]), s, self.labels, self.n_sink, self.window,
                                              evict, pick)
                tol = h * np.abs(o) + (w + 2 * (self.d + 3) * U * size + (s + n + 20) * U) * mass
                err = np.abs(f64(out[at:at + n])[pick] - o)
                assert np.isfinite(err).all(), f"sequence {i} ({s}, {n}): not finite"
                worst = max(worst, float((err / tol).max()))
            at += n
        assert worst <= 1, f"{worst:.3f} of the bound"


# labels, query heads a group, sink, window, sequences (start, new)
COUNTS = [
    ([0, 1], 1, 4, 28, [(0, 1), (1, 1), (15, 1), (16, 1), (17, 2), (63, 1), (64, 3), (200, 1)]),
    ([0, 1], 4, 4, 60, [(100, 4), (5, 4), (64, 4), (0, 3)]),
    ([1, 0, 1], 7, 0, 77, [(500, 5), (3, 2), (76, 9), (78, 1)]),
    ([0, 1], 16, 16, 64, [(129, 2), (63, 7)]),
    ([0, 1], 4, 3, 40, [(30, 100), (0, 0), (0, 70), (300, 33)]),
    ([0, 1], 7, 70, 130, [(10, 300), (900, 150), (199, 1), (201, 64)]),
    ([0, 1], 1, 64, 256, [(1000, 513), (0, 700), (64, 65)]),
    ([1], 2, 0, 1, [(9, 40), (0, 5)]),
    ([1, 1], 3, 200, 9, [(100, 300), (250, 20), (0, 1)]),
    ([0], 5, 4, 4, [(2047, 129), (4096, 31), (0, 64)]),
    ([0, 1], 2, 4, 1000, [(3000, 1), (5000, 3), (2, 2)]),
]


@pytest.mark.parametrize("case", COUNTS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("evict", [False, True])
def test_every_visible_key_counts_once(case, d, evict):
    labels, gs, n_sink, window, seqs = case
    run = Run(labels, gs, d, n_sink, window, seqs, count=True)
    run.check_counts(run.extend(F32, evict=evict), evict)


@pytest.mark.parametrize("d", [64, 128])
def test_counts_of_long_prefixes_and_many_sequences(d):
    run = Run([0, 1], 4, d, 16, 300, [(20000, 3), (40, 2), (7000, 1)], count=True, seed=2)
    run.check_counts(run.extend(F32))
    run = Run([0, 1], 2, d, 4, 28, [(37 * i % 400, i % 7) for i in range(150)], count=True, seed=3)
    run.check_counts(run.extend(F32))
    run = Run([0], 2, d, 4, 28, [(9000, 260)], count=True, seed=4)
    run.check_counts(run.extend(F32))


@pytest.mark.parametrize("d", [64, 128])
def test_more_sequences_than_a_launch_plans(d):
    run = Run([1, 0], 1, d, 2, 14, [(5 * i % 40, 1 + i % 3) for i in range(1300)], count=True, seed=5)
    run.check_counts(run.extend(F32))


VALUES = [
    ([0, 1], 4, 4, 60, [(300, 5), (0, 3), (77, 1)]),
    ([0, 1], 7, 16, 200, [(1500, 17), (100, 40)]),
    ([0, 1], 2, 4, 100, [(700, 300), (0, 257)]),
    ([0], 1, 4, 4, [(600, 200)]),
]


@pytest.mark.parametrize("case", VALUES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_values(case, d, out_dtype):
    labels, gs, n_sink, window, seqs = case
    run = Run(labels, gs, d, n_sink, window, seqs, seed=6)
    for evict in (False, True):
        run.check_values(run.extend(out_dtype, evict=evict), evict)


@pytest.mark.parametrize("d", [64, 128])
def test_values_of_fp32_rows(d):
    for i, (labels, gs, n_sink, window, seqs) in enumerate(VALUES[:3]):
        run = Run(labels, gs, d, n_sink, window, seqs, dtype=F32, seed=7)
        run.check_values(run.extend(evict=bool(i & 1)), bool(i & 1))


@pytest.mark.parametrize("shape", [(17, 2, 7), (200, 1, 4), (3, 6, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_far_apart(shape, d):
    """Weights that move to new maxima along the sequence, and scores of some hundreds."""
    n, _, gs = shape
    run = Run([0, 1], gs, d, 4, 500, [(900, n)], seed=8)
    ramp = torch.linspace(0, 6, 900 + n)[:, None, None]
    base = torch.randn(1, 2, d, generator=torch.Generator().manual_seed(1))
    run.k = [(run.k[0] * 0.3 + base * ramp).to(BF)]
    run.q = [(run.q[0] * 0.5 + base.repeat_interleave(gs, 1)).to(BF)]
    run.fill()
    for dt in (BF, F32):
        run.check_values(run.extend(dt))


@pytest.mark.parametrize("n, gs", [(3, 2), (5, 7), (40, 4), (200, 2), (300, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_seen_has_no_influence(n, gs, d):
    """K and V of late tokens that are not finite leave the queries before them alone (and reach those behind); window
    tokens that are not finite leave the queries alone whose window has moved on."""
    run = Run([0, 1], gs, d, 4, 24, [(100, n)], seed=9)
    want = {dt: run.extend(dt) for dt in (BF, F32)}
    at = n // 2
    for value, which in ((NAN, "v"), (float("inf"), "v"), (NAN, "k"), (-float("inf"), "v")):
        bad = Run([0, 1], gs, d, 4, 24, [(100, n)], seed=9)
        getattr(bad, which)[0][100 + at:, :, 3] = value
        for dt in (BF, F32):
            got = bad.extend(dt)
            assert np.array_equal(bits(got[:at]), bits(want[dt][:at])), (value, which, dt)
            if which == "v":
                assert not torch.isfinite(got[at:, :, 3]).any()
                assert np.array_equal(bits(got[at:, :, 4:]), bits(want[dt][at:, :, 4:]))
            else:
                assert torch.isnan(got[at:]).all()
    # position 80 (in the ring): seen by queries up to 80 + 23 = 103, that is up to t = 3
    bad = Run([0, 1], gs, d, 4, 24, [(100, n)], seed=9)
    bad.v[0][80, 1] = NAN
    bad.fill()
    got = bad.extend()
    assert torch.isnan(got[:4, gs:]).all() and np.array_equal(bits(got[4:]), bits(want[BF][4:]))
    assert np.array_equal(bits(got[:, :gs]), bits(want[BF][:, :gs]))


@pytest.mark.parametrize("n", [2, 33])
def test_queries_keep_to_themselves(n):
    run = Run([0, 1], 4, 128, 4, 24, [(100, n)], seed=10)
    want = run.extend()
    run.q[0][1, 2] = NAN
    got = run.extend()
    same = (bits(got) == bits(want)).all(-1)
    assert not same[1, 2] and same.sum() == n * 8 - 1


@pytest.mark.parametrize("chunk", [1, 16, 100, 130])
@pytest.mark.parametrize("evict", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_after_chunk_is_a_prefill(chunk, evict, d):
    """The paper's chunked prefill: rows as the prefill's (both within their rounding of the same values), caches bit for
    bit as of one append."""
    total, labels, gs, n_sink, window = 300, [0, 1, 1], 3, 8, 50
    run = Run(labels, gs, d, n_sink, window, [(0, total)], seed=11)
    q, k, v, _ = run.packed(0)
    out = torch.empty_like(q)
    for s in range(0, total, chunk):
        e = min(s + chunk, total)
        aoh_extend(q[None, s:e], k[None, s:e], v[None, s:e], labels, i32([s]), run.full, run.ring, n_sink, window, evict=evict,
                   out=out[None, s:e])
    want = (aoh_prefill_chunked(q[None], k[None], v[None], labels, n_sink, window, chunk) if evict else
            aoh_prefill(q[None], k[None], v[None], labels, n_sink, window))[0]
    assert (out.float() - want.float()).abs().max() < 2e-2
    if not evict or chunk >= total:
        run.check_values(out, evict)
    whole = Run(labels, gs, d, n_sink, window, [(0, total)], seed=11)
    whole.append(0, 0, total, whole.full, whole.ring)
    for a, b in zip(run.tensors(), whole.tensors()):
        assert np.array_equal(bits(a), bits(b))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_dense_batches_and_their_append(d, dtype):
    """A dense batch with strides of its own gives the packed call's rows; append writes what aoh_kv_append writes, without
    it nothing is written."""
    seqs = [(40, 9), (0, 9), (133, 9)]
    run = Run([1, 0, 0], 3, d, 5, 30, seqs, dtype=dtype, seed=12)
    before = [bits(t) for t in run.tensors()]
    want = run.extend()
    assert all(np.array_equal(x, bits(t)) for x, t in zip(before, run.tensors()))
    q, k, v, _ = (x.unflatten(0, (3, 9)) if x.dim() == 3 else x for x in run.packed(0))
    out = torch.full((3, 9, 2 * run.hq, d), 7.0, dtype=dtype, device=DEV)
    aoh_extend(q, k, v, run.labels, i32(run.starts), run.full, run.ring, 5, 30, append=True, out=out[:, :, ::2])
    assert np.array_equal(bits(out[:, :, ::2].flatten(0, 1)), bits(want)) and (out[:, :, 1::2] == 7).all()
    other = Run([1, 0, 0], 3, d, 5, 30, seqs, dtype=dtype, seed=12)
    for i, (s, n) in enumerate(seqs):
        other.append(i, s, s + n, other.full, other.ring)
    for a, b in zip(run.tensors(), other.tensors()):
        assert np.array_equal(bits(a), bits(b))
    # packed, with the append
    third = Run([1, 0, 0], 3, d, 5, 30, seqs, dtype=dtype, seed=12)
    assert np.array_equal(bits(third.extend(append=True)), bits(want))
    for a, b in zip(third.tensors(), other.tensors()):
        assert np.array_equal(bits(a), bits(b))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [2, 40])
def test_starts_and_pages_outside_the_caches(n, dtype):
    """Sequences with a start that is none are left out; pages that are not mapped are not seen, and positions beyond the
    block table neither."""
    d, gs = 64, 4
    run = Run([0, 1], gs, d, 4, 28, [(64, n)] * 5, dtype=dtype, seed=13, count=True)
    q, k, v, _ = (x.unflatten(0, (5, n)) if x.dim() == 3 else x for x in run.packed(0))
    run.table[2, 1] = -1
    run.table[3, 2] = run.full.k.shape[0]
    full = PagedCache(run.full.k, run.full.v, run.table[:, :3].contiguous())  # 48 positions
    out = torch.full((5, n, 2 * gs, d), 7.0, dtype=F32, device=DEV)
    aoh_extend(q, k, v, run.labels, i32([-1, (1 << 30) + 1, 64, 64, 64]), full, run.ring, 4, 28, append=False, out=out)
    assert (out[:2] == 7).all()
    for i, pages in ((2, [0, 2]), (3, [0, 1]), (4, [0, 1, 2])):
        seen = torch.cat([run.v[i][16 * p:16 * p + 16, 0] for p in pages]).double().sum(0)
        for t in range(n):
            ones = seen + run.v[i][64:65 + t, 0].double().sum(0)
            got = out[i, t, :gs].cpu().double() * (16 * len(pages) + t + 1)
            assert (got - ones).abs().max() < 0.01, (i, t)


@pytest.mark.parametrize("n, start", [(2, 3000), (60, 500), (300, 100)])
def test_streams_and_graphs(n, start):
    """Replays of one captured call follow its inputs and starts; calls of two streams run side by side."""
    run = Run([0, 1], 4, 128, 4, 200, [(start, n)] * 2, seed=14)
    q, k, v, _ = (x.unflatten(0, (2, n)).contiguous() if x.dim() == 3 else x for x in run.packed(0))
    starts, out = i32([start] * 2), torch.empty_like(q)
    args = (run.labels, starts, run.full, run.ring, 4, 200)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        aoh_extend(q, k, v, *args, append=False, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        aoh_extend(q, k, v, *args, append=False, out=out)
    for i in range(4):
        q.mul_(0.75)
        starts.fill_(start - 7 * i)
        g.replay()
        torch.cuda.synchronize()
        want = aoh_extend(q, k, v, *args, append=False)
        torch.cuda.synchronize()
        assert np.array_equal(bits(out), bits(want)), i
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [aoh_extend(q, k, v, *args, append=False, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(np.array_equal(bits(x), bits(want)) for x in got)


def test_a_cache_beyond_four_gigabytes():
    d, pages = 128, 1 << 17
    run = Run([0] * 8, 2, d, 4, 28, [(100, 3)], seed=15, count=True)
    k, v = (torch.zeros((pages, 8, *s), dtype=BF, device=DEV) for s in ((16, d), (d, 16)))
    table = torch.arange(pages - 9, pages, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    run.full = PagedCache(k, v, table)
    run.append(0, 0, 100, run.full, None)
    run.check_counts(run.extend(F32))
    run.check_counts(run.extend(F32, append=True))
    assert np.array_equal(bits(k[pages - 7, :, 4:7].transpose(0, 1)), bits(run.k[0][100:103]))


@pytest.mark.parametrize("d, out_dtype", [(128, BF), (64, F32)])
def test_sequences_that_overlap_need_no_more_room_than_there_is(d, out_dtype):
    """Offsets that are not ascending: 32 times all 600 rows, for which the workspace has no room."""
    run = Run([0, 1], 4, d, 4, 28, [(0, 600)] + [(0, 0)] * 63)
    q, k, v, _ = run.packed(0)
    cu = i32([0, 600] * 32 + [600])
    ws = torch.full((aoh_extend_workspace_bytes(64, 600, 8, 2, d) + 4096,), 5, dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, 7.0, dtype=out_dtype, device=DEV)
    aoh_extend_varlen(q, k, v, cu, 600, run.labels, None, run.full, run.ring, 4, 28, append=False, out=out, workspace=ws[:-4096])
    assert (out == 7).all() and (ws[-4096:] == 5).all()
