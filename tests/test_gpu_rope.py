"""Head norms and position rotation against the oracle in extended precision, and the appends that apply them against
the two calls that they stand for.

Bound of one output value z with partner values y_a, y_b (u = 2^-24, half a step of fp32; h half a step of the rows'
dtype): h |z| for the last rounding; the fp32 part before it
  norm    the mean of squares: a chain of at most 8 products and sums, 5 tree sums, the factor, the eps: 15 u, half of it
          behind the root; root, reciprocal, two products: at most 5 u (the root and the reciprocal within an ulp):
          13 u of y
  angle   |a| 2^-51 (two fp64 products and the constant 1 / 2 pi, each within 2^-53 of |a|), for bf16 rows the fraction of a
          turn in fp32 (pi u) and the functions (4 ulps, 4 u at most), their product with the scale (u): 9 u scale
  sum     a product and a fused sum: 2 u of |y_a c| + |y_b s|
so |error| <= h |z| (1 + u) + (24 u + 2^-51 |a|) (|y_a| + |y_b|) max(1, scale) altogether."""
import numpy as np
import pytest
import torch

import synth
from oracle import rope as oracle
from paper_2608_06849_amd import (PagedCache, RingCache, Rope, aoh_kv_append, aoh_kv_append_rope,
                                  aoh_kv_append_rope_varlen, aoh_qk_rope)
from tests.helpers import bits, f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def draw(shape, seed, name, dtype):
    return torch.from_numpy(synth.gaussian(shape, seed, name)).to(dtype).to(DEV)


def freqs(pairs, theta=1e6):
    return torch.from_numpy((theta ** (-np.arange(pairs) / pairs)).astype(np.float32)).to(DEV)


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(DEV)


def held(got, x, weight, eps, rope, pos, what):
    """`got` within the bound of the oracle's rows x [B, T, H, D] at positions pos [axes, B * T]."""
    rows = f64(x).reshape(-1, *x.shape[2:])
    y = oracle.norm(rows, None if weight is None else f64(weight), eps)
    d = rows.shape[-1]
    if rope is None:
        z, part, far = y, np.abs(y), 0.0
    else:
        f = rope.inv_freq.cpu().numpy()
        ang = oracle.angles(pos, f, list(rope.axis) if rope.axis else None)
        z = oracle.rotate(y, ang, rope.interleaved, rope.scale)
        pair, mate, _ = oracle.partners(d, len(f), rope.interleaved)
        part = np.abs(y) + np.where(pair >= 0, np.abs(y[..., mate]), 0)
        far = np.where(pair >= 0, np.abs(ang)[:, pair], 0)[:, None] * 2.0 ** -51
        part = part * max(1.0, abs(rope.scale))
    h = torch.finfo(x.dtype).eps / 2
    tol = h * np.abs(z) * (1 + U) + (24 * U + far) * part
    err = np.abs(f64(got).reshape(z.shape) - z)
    worst = float((err / np.maximum(tol, 1e-300)).max())
    assert worst <= 1, f"{what}: {worst:.3f} of the bound"


SHAPES = [(1, 1, 28, 4), (3, 7, 5, 1), (2, 33, 32, 8), (70, 1, 8, 8), (1, 300, 16, 16)]
# pairs (0: no rotation), interleaved, axes, norms, scale
FORMS = [(64, False, 1, "qk", 1.0), (64, True, 1, "", 1.0), (32, False, 1, "q", 1.25), (13, False, 3, "k", 1.0),
         (1, True, 1, "", 0.5), (8, False, 1, "", 1.0), (31, True, 3, "qk", 1.0), (0, False, 1, "qk", 1.0)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("d, dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
def test_rows_against_the_oracle(shape, form, d, dtype):
    (b, t, hq, hkv), (pairs, inter, axes, norms, scale) = shape, form
    pairs = min(pairs, d // 2)
    x = draw((b, t, hq + hkv, d), 5, f"x{shape}{form}", dtype)
    q, k = x[:, :, :hq], x[:, :, hq:]  # slices of one tensor
    w = [(1 + 0.3 * draw((d,), 5, f"w{i}", F32)).to(dtype if t % 2 else F32) if n in norms else None for i, n in enumerate("qk")]
    start = i32([(977 * i) % 5000 for i in range(b)])
    rope = pos = None
    if pairs:
        axis = [i % axes for i in range(pairs)] if axes > 1 else None
        rope = Rope(freqs(pairs), axis=axis, interleaved=inter, scale=scale)
        where = (f64(start).astype(int)[:, None] + np.arange(t)).reshape(1, -1)
        if axes > 1:
            where = np.stack([1000 * where[0] + 7, where[0] // 3 - 50, where[0] % 23])
            pos = i32(where).view(axes, b, t)
    before = bits(x)
    gq, gk = aoh_qk_rope(q, k, rope, q_norm=w[0], k_norm=w[1], eps=1e-5, positions=pos, start_pos=start)
    held(gq, q, w[0], 1e-5, rope, where if pairs else None, "q")
    held(gk, k, w[1], 1e-5, rope, where if pairs else None, "k")
    assert np.array_equal(bits(x), before)
    # in place, and each alone: the same bits
    one, _ = aoh_qk_rope(q, None, rope, q_norm=w[0], eps=1e-5, positions=pos, start_pos=start) if pairs or w[0] is not None else (gq, 0)
    _, two = aoh_qk_rope(None, k, rope, k_norm=w[1], eps=1e-5, positions=pos, start_pos=start) if pairs or w[1] is not None else (0, gk)
    aoh_qk_rope(q, k, rope, q_norm=w[0], k_norm=w[1], eps=1e-5, positions=pos, start_pos=start, q_out=q, k_out=k)
    for a in (one, q):
        assert np.array_equal(bits(a), bits(gq))
    for a in (two, k):
        assert np.array_equal(bits(a), bits(gk))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("base", [0, 1 << 20, (1 << 31) - 40, -(1 << 31)])
def test_far_positions(dtype, base):
    q = draw((1, 37, 2, 128), 6, "far", dtype)
    rope = Rope(freqs(64))
    pos = base + np.arange(37)[None]
    got, _ = aoh_qk_rope(q, None, rope, positions=i32(pos).view(1, 1, 37))
    held(got, q, None, 0, rope, pos, f"from {base}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_keep_to_themselves(dtype):
    """Values that are not finite stay in their row, those that are not rotated in their value, zeros stay zeros."""
    q = draw((1, 20, 6, 64), 7, "q", dtype)
    want, _ = aoh_qk_rope(q, None, Rope(freqs(16)))
    bad = q.clone()
    bad[0, 3, 1, 5] = float("nan")
    bad[0, 7, 2, 40] = float("inf")
    bad[0, 9, 4] = 0
    got, _ = aoh_qk_rope(bad, None, Rope(freqs(16)))
    diff = bits(got) != bits(want)
    expect = np.zeros_like(diff)
    expect[0, 3, 1, [5, 21]] = expect[0, 7, 2, 40] = True
    assert (diff & ~expect).any(axis=(1, 3))[0].tolist() == [False] * 4 + [True] + [False]  # only the zeroed row besides
    assert torch.isnan(got[0, 3, 1, [5, 21]]).all() and torch.isinf(got[0, 7, 2, 40]) and (got[0, 9, 4] == 0).all()
    w = torch.ones(64, dtype=dtype, device=DEV)
    normed, _ = aoh_qk_rope(bad, None, None, q_norm=w, eps=1e-6)
    clean, _ = aoh_qk_rope(q, None, None, q_norm=w, eps=1e-6)
    same = (bits(normed) == bits(clean)).all(-1)[0]
    assert not same[3, 1] and not same[7, 2] and same.sum() == 20 * 6 - 3 and (normed[0, 9, 4] == 0).all()


class Caches:
    """Caches filled with NaN bits; spare pages stand between the sequences' ones."""

    def __init__(self, labels, b, tokens, d, n_sink, window, dtype, token_major=False, seed=1):
        pages = max(1, (tokens + 15) // 16)
        bt = torch.from_numpy(synth.page_permutation(b * pages + 3, seed, "pages")[:b * pages].reshape(b, pages).astype(np.int32))
        self.labels, self.n_sink, self.window = labels, n_sink, window
        self.full = PagedCache.allocate(b * pages + 3, labels.count(0), d, dtype, bt, v_token_major=token_major) if 0 in labels else None
        self.ring = RingCache.allocate(b, labels.count(1), n_sink, window, d, dtype) if 1 in labels else None
        for t in self.tensors():
            t.fill_(float("nan"))

    def tensors(self):
        return [t for c in (self.full, self.ring) if c is not None for t in (c.k, c.v)]

    @property
    def args(self):
        return self.full, self.ring, self.n_sink, self.window

    def same(self, other):
        for a, b in zip(self.tensors(), other.tensors()):
            assert np.array_equal(bits(a), bits(b))


# labels, batch, new tokens, starts (first ones repeated), sink, window
APPENDS = [([0, 1, 0, 1], 1, 1, [4092], 4, 60), ([0, 1], 5, 1, [0, 15, 16, 63, 200], 4, 28), ([0, 0, 0], 3, 37, [0, 5, 16], 4, 28),
           ([1, 1], 3, 50, [0, 3, 100], 0, 7), ([0, 1, 1], 2, 200, [9, 32], 16, 64), ([1], 2, 16, [16, 48], 16, 32),
           ([0, 1], 70, 2, [14, 15, 31], 3, 40)]


@pytest.mark.parametrize("case", APPENDS, ids=str)
@pytest.mark.parametrize("d, dtype", [(128, BF), (64, BF), (128, F32), (64, F32)])
def test_append_is_the_two_calls(case, d, dtype):
    labels, b, n, starts, n_sink, window = case
    hkv, hq = len(labels), 3 * len(labels)
    starts = [starts[i % len(starts)] for i in range(b)]
    x = draw((b, n, hq + 2 * hkv, d), 8, f"x{case}", dtype)
    q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    rope, start = Rope(freqs(d // 2)), i32(starts)
    w = [(1 + 0.3 * draw((d,), 8, f"w{i}", F32)).to(dtype) for i in range(2)]
    top = max(starts) + n
    for norms, pos, major in ((w, None, False), ([None, None], i32(np.arange(b * n) * 5 + 3).view(1, b, n), True)):
        one, two = (Caches(labels, b, top, d, n_sink, window, dtype, major) for _ in range(2))
        kw = dict(q_norm=norms[0], k_norm=norms[1], eps=1e-6, positions=pos)
        got = aoh_kv_append_rope(q, k, v, rope, labels, start, *one.args, **kw)
        wq, wk = aoh_qk_rope(q, k, rope, start_pos=start, **kw)
        aoh_kv_append(wk, v, labels, start, *two.args)
        assert np.array_equal(bits(got), bits(wq))
        one.same(two)
        # without queries, then without anything but the copy
        three, four, five = (Caches(labels, b, top, d, n_sink, window, dtype, major) for _ in range(3))
        kw.pop("q_norm")
        assert aoh_kv_append_rope(None, k, v, rope, labels, start, *three.args, **kw) is None
        three.same(two)
        raw = k.clone()
        raw.view(torch.int16 if dtype == BF else torch.int32)[0, 0, 0, :3] = 0x7F81 if dtype == BF else 0x7F800001  # a signalling NaN
        aoh_kv_append_rope(None, raw, v, None, labels, start, *four.args)
        aoh_kv_append(raw, v, labels, start, *five.args)
        four.same(five)


@pytest.mark.parametrize("d, dtype", [(128, BF), (64, BF), (128, F32)])
def test_packed_append_is_the_dense_calls(d, dtype):
    labels, n_sink, window, hq = [0, 1, 0], 4, 28, 6
    lens, starts = [5, 0, 1, 40, 17, 16], [3, 9, 31, 0, 8, 32]
    b, total = len(lens), sum(lens) + 4  # rows behind the last sequence
    cu = np.concatenate([[0], np.cumsum(lens)])
    x = draw((total, hq + 6, d), 9, "x", dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + 3], x[:, hq + 3:]
    axis = [i % 2 for i in range(d // 2)]
    rope, pos = Rope(freqs(d // 2), axis=axis), i32(np.stack([np.arange(total) * 3, 1000 - np.arange(total)]))
    w = (1 + 0.3 * draw((d,), 9, "w", F32)).to(dtype)
    one, two = (Caches(labels, b, 64, d, n_sink, window, dtype) for _ in range(2))
    out = torch.full((total, hq, d), 7.0, dtype=dtype, device=DEV)
    got = aoh_kv_append_rope_varlen(q, k, v, i32(cu), max(lens), rope, labels, i32(starts), *one.args, k_norm=w, positions=pos,
                                    q_out=out)
    assert got is out and (out[cu[-1]:] == 7).all()
    for i, n in enumerate(lens):
        if n == 0:
            continue
        r = slice(cu[i], cu[i + 1])
        table, ring = two.full.rows(i, i + 1), RingCache(two.ring.k[i:i + 1], two.ring.v[i:i + 1], two.ring.capacity)
        wq = aoh_kv_append_rope(q[None, r], k[None, r], v[None, r], rope, labels, i32(starts[i:i + 1]), table, ring, n_sink, window,
                                k_norm=w, positions=pos[:, r].contiguous().view(2, 1, n))
        assert np.array_equal(bits(out[r]), bits(wq[0]))
    one.same(two)


def test_starts_and_pages_outside_the_caches_write_nothing_there():
    labels, d, n = [0, 1], 64, 20
    q, k, v = (draw((5, n, h, d), 10, f"x{h}{i}", BF) for i, h in enumerate((4, 2, 2)))
    rope = Rope(freqs(32))
    one, two = (Caches(labels, 5, 48, d, 4, 28, BF) for _ in range(2))
    for c in (one, two):
        c.full.block_table[3, 1] = -1
        c.full.block_table[4, 0] = c.full.k.shape[0]
    starts = [-1, (1 << 30) + 1, 40, 10, 0]
    out = torch.full((5, n, 4, d), 7.0, dtype=BF, device=DEV)
    aoh_kv_append_rope(q, k, v, rope, labels, i32(starts), *one.args, q_out=out)
    assert (out[:2] == 7).all()
    wq, wk = aoh_qk_rope(q, k, rope, start_pos=i32(starts))
    assert np.array_equal(bits(out[2:]), bits(wq[2:]))
    aoh_kv_append(wk, v, labels, i32([-1, -1] + starts[2:]), *two.args)
    one.same(two)


def test_captured_and_on_a_stream():
    """Replays see new inputs and positions; a call on a given stream gives the same."""
    labels, d, b = [0, 1], 128, 3
    rope, start = Rope(freqs(64)), i32([5, 15, 90])
    x = draw((b, 1, 8, d), 11, "x", BF)
    q, k, v = x[:, :, :4], x[:, :, 4:6], x[:, :, 6:]
    c = Caches(labels, b, 200, d, 4, 60, BF)
    out, (qo, ko) = torch.empty_like(q), (torch.empty_like(q), torch.empty_like(k))
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        aoh_kv_append_rope(q, k, v, rope, labels, start, *c.args, q_out=out)
        aoh_qk_rope(q, k, rope, start_pos=start, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        aoh_kv_append_rope(q, k, v, rope, labels, start, *c.args, q_out=out)
        aoh_qk_rope(q, k, rope, start_pos=start, q_out=qo, k_out=ko)
    want = Caches(labels, b, 200, d, 4, 60, BF)
    for t, u in zip(c.tensors(), want.tensors()):
        u.copy_(t)
    for step in range(4):
        x.copy_(draw((b, 1, 8, d), 12 + step, "x", BF))
        g.replay()
        torch.cuda.synchronize()
        w = aoh_kv_append_rope(q, k, v, rope, labels, start, *want.args, stream=side)
        side.synchronize()
        assert np.array_equal(bits(out), bits(w)) and np.array_equal(bits(qo), bits(w))
        c.same(want)
        start += 1


def test_a_cache_beyond_four_gigabytes():
    labels, d, pages = [0, 0, 0, 0, 0, 0, 0, 0], 128, 1 << 17
    table = i32([[pages - 1, pages - 2]])
    full = PagedCache(*(torch.zeros((pages, 8, *s), dtype=BF, device=DEV) for s in ((16, d), (d, 16))), table)
    k, v = (draw((1, 20, 8, d), 13, n, BF) for n in "kv")
    rope = Rope(freqs(64))
    aoh_kv_append_rope(None, k, v, rope, labels, i32([3]), full, None, 4, 28)
    _, wk = aoh_qk_rope(None, k, rope, start_pos=i32([3]))
    assert np.array_equal(bits(full.k[pages - 1, :, 3:].transpose(0, 1)), bits(wk[0, :13]))
    assert np.array_equal(bits(full.v[pages - 2, :, :, :7].permute(2, 0, 1)), bits(v[0, 13:]))
    assert int((full.k.view(torch.int16) != 0).any(-1).sum()) == 160
