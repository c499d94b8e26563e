"""Conversations as a server runs them: packed prompts, drafted tokens and single steps one after another over the same
caches.  Every answer is held to the float64 oracle on all tokens so far; what the caches hold is seen only through the
calls that read it, and they hold NaN at first."""
import numpy as np
import pytest
import torch

from oracle import attention, extend as oracle
from paper_2608_06849_amd import (PagedCache, PagedCacheQ8, RingCache, RingCacheQ8, Rope, aoh_decode, aoh_decode_step_q8,
                                  aoh_decode_workspace_bytes, aoh_extend, aoh_extend_varlen, aoh_kv_append_q8, aoh_kv_append_rope,
                                  aoh_kv_read_q8, aoh_qk_rope)
from tests.helpers import assert_parity, bits, f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
B, HQ, LABELS, SINK, WINDOW, EPS = 3, 8, [0, 1], 4, 60, 1e-5
HKV = len(LABELS)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Talk:
    """Rows of a projection, normed and turned by aoh_qk_rope, and all keys and values so far."""

    def __init__(self, d, dtype, seed):
        self.d, self.dtype = d, dtype
        self.g = torch.Generator().manual_seed(seed)
        self.rope = Rope(10000.0 ** (-torch.arange(d // 4, device=DEV).float() / (d // 4)))
        self.norms = dict(q_norm=1 + 0.3 * self.draw(d), k_norm=1 + 0.3 * self.draw(d), eps=EPS)
        self.k, self.v = ([[] for _ in range(B)] for _ in range(2))
        self.lens = [0] * B

    def draw(self, *shape):
        return torch.randn(shape, generator=self.g).to(self.dtype).to(DEV)

    def caches(self, paged, ring):
        pages = 24
        table = torch.randperm(B * pages + 2, generator=self.g)[:B * pages].view(B, pages).int().to(DEV)
        full, ring = paged.allocate(B * pages + 2, 1, self.d, *([self.dtype] if paged is PagedCache else [torch.int8]), table), \
            ring.allocate(B, 1, SINK, WINDOW, self.d, self.dtype if ring is RingCache else torch.int8)
        return full, ring

    def rows(self, n):
        """q, k, v of n tokens, slices of one projection's output."""
        x = self.draw(1, n, HQ + 2 * HKV, self.d)
        return x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]

    def step(self, q, full, ring):
        ws = torch.empty(aoh_decode_workspace_bytes(B, HQ, self.d, full.block_table.shape[1], ring.capacity), dtype=torch.uint8, device=DEV)
        return aoh_decode(q.contiguous(), full, ring, LABELS, i32(self.lens), SINK, WINDOW, workspace=ws)

    def remember(self, i, k, v):
        self.k[i].append(f64(k))
        self.v[i].append(f64(v))
        self.lens[i] += len(k)

    def sequence(self, i):
        return np.concatenate(self.k[i]), np.concatenate(self.v[i])

    def check_new(self, out, q, news):
        """The bound of tests/test_gpu_extend.py: rounding of the result and of bf16 weights, fp32 scores and sums."""
        at, h, w = 0, torch.finfo(self.dtype).eps / 2, 2.0 ** -8 if self.dtype == BF else 0.0
        for i, n in enumerate(news):
            if n:
                k, v = self.sequence(i)
                o, mass, size = oracle.extend(f64(q[at:at + n]), k, v, len(k) - n, LABELS, SINK, WINDOW, False)
                tol = h * np.abs(o) + (w + 2 * (self.d + 3) * U * size + (len(k) + 20) * U) * mass
                worst = float((np.abs(f64(out[at:at + n]) - o) / tol).max())
                assert worst <= 1, f"sequence {i}, {n} after {len(k) - n}: {worst:.3f} of the bound"
            at += n

    def check_step(self, out, q):
        if self.dtype == F32:  # the same bound
            return self.check_new(out, q, [1] * B)
        for i in range(B):
            k, v = self.sequence(i)
            assert_parity(out[i:i + 1].cpu(), attention.decode(f64(q[i:i + 1]), k[None], v[None], [len(k)], LABELS, SINK, WINDOW),
                          self.dtype, f"sequence {i} at {len(k)}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompts_drafts_and_steps(d, dtype):
    t = Talk(d, dtype, 40 + d)
    full, ring = t.caches(PagedCache, RingCache)
    for x in (full.k, full.v, ring.k, ring.v):
        x.fill_(float("nan"))
    for turn in range(3):
        # messages of different lengths, one of them empty: positions go on where each sequence stands
        news = [[37, 0, 90], [1, 64, 33], [16, 75, 0]][turn]
        cu = i32(np.concatenate([[0], np.cumsum(news)]).tolist())
        q, k, v = t.rows(sum(news))
        pos = i32(np.concatenate([np.arange(t.lens[i], t.lens[i] + n) for i, n in enumerate(news)]).tolist()).view(1, 1, -1)
        q, k = aoh_qk_rope(q, k, t.rope, positions=pos, **t.norms)
        out = aoh_extend_varlen(q[0], k[0], v[0], cu, max(news), LABELS, i32(t.lens), full, ring, SINK, WINDOW)
        for i in range(B):
            a, b = int(cu[i]), int(cu[i + 1])
            t.remember(i, k[0, a:b], v[0, a:b])
        t.check_new(out, q[0], news)
        # four drafted tokens of each sequence are verified, two are taken
        q, k, v = (x.view(B, 4, -1, d) for x in t.rows(4 * B))
        before = i32(t.lens)
        q, k = aoh_qk_rope(q, k, t.rope, start_pos=before, **t.norms)
        out = aoh_extend(q, k, v, LABELS, before, full, ring, SINK, WINDOW, append=False)
        for i in range(B):
            t.remember(i, k[i], v[i])
        t.check_new(out.reshape(-1, HQ, d), q.reshape(-1, HQ, d), [4] * B)
        for i in range(B):
            t.k[i][-1], t.v[i][-1] = t.k[i][-1][:2], t.v[i][-1][:2]
            t.lens[i] -= 2
        aoh_extend(q[:, :2], k[:, :2], v[:, :2], LABELS, before, full, ring, SINK, WINDOW)
        # single tokens: norm, rotation and append in one call, then the step
        for _ in range(3):
            q, k, v = (x.view(B, 1, -1, d) for x in t.rows(B))
            before = i32(t.lens)
            turned = aoh_kv_append_rope(q, k, v, t.rope, LABELS, before, full, ring, SINK, WINDOW, **t.norms)
            same = aoh_qk_rope(q, k, t.rope, start_pos=before, **t.norms)
            assert np.array_equal(bits(turned), bits(same[0]))
            for i in range(B):
                t.remember(i, same[1][i], v[i])
            t.check_step(t.step(turned[:, 0], full, ring), turned[:, 0])


@pytest.mark.parametrize("d", [64, 128])
def test_a_captured_step(d):
    """Norm, rotation, append and attention of single tokens, captured once: positions come from the lengths, so that each
    replay is the next token."""
    t = Talk(d, BF, 70 + d)
    full, ring = t.caches(PagedCache, RingCache)
    news = [30, 61, 17]
    cu = i32(np.concatenate([[0], np.cumsum(news)]).tolist())
    q, k, v = t.rows(sum(news))
    pos = i32(np.concatenate([np.arange(n) for n in news]).tolist()).view(1, 1, -1)
    q, k = aoh_qk_rope(q, k, t.rope, positions=pos, **t.norms)
    aoh_extend_varlen(q[0], k[0], v[0], cu, max(news), LABELS, None, full, ring, SINK, WINDOW)
    for i in range(B):
        t.remember(i, k[0, cu[i]:cu[i + 1]], v[0, cu[i]:cu[i + 1]])
    x = torch.zeros((B, 1, HQ + 2 * HKV, d), dtype=BF, device=DEV)
    q, k, v = x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]
    lens = i32(t.lens)
    turned, out = torch.empty((B, 1, HQ, d), dtype=BF, device=DEV), torch.empty((B, 1, HQ, d), dtype=BF, device=DEV)
    keys = torch.empty((B, 1, HKV, d), dtype=BF, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        # an answer by aoh_extend over the caches and the token, then the same token into the caches
        aoh_qk_rope(q, k, t.rope, start_pos=lens, q_out=turned, k_out=keys, **t.norms)
        aoh_extend(turned, keys, v, LABELS, lens, full, ring, SINK, WINDOW, append=False, out=out)
        aoh_kv_append_rope(q, k, v, t.rope, LABELS, lens, full, ring, SINK, WINDOW, q_out=turned, **t.norms)
        lens += 1
    for _ in range(6):
        x.copy_(t.draw(*x.shape))
        before = i32(t.lens)
        want_q, want_k = aoh_qk_rope(q, k, t.rope, start_pos=before, **t.norms)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(turned), bits(want_q)) and np.array_equal(bits(keys), bits(want_k))
        for i in range(B):
            t.remember(i, want_k[i], v[i])
        assert lens.tolist() == t.lens
        t.check_new(out[:, 0], turned[:, 0], [1] * B)
        # the caches hold the token too
        t.check_step(t.step(turned[:, 0], full, ring), turned[:, 0])


@pytest.mark.parametrize("d", [64, 128])
def test_turned_keys_in_eight_bit_caches(d):
    """Keys of aoh_qk_rope in 8-bit caches: the steps answer as on what those caches hold."""
    t = Talk(d, BF, 90 + d)
    full, ring = t.caches(PagedCacheQ8, RingCacheQ8)
    n = 50
    q, k, v = (x.view(B, n, -1, d) for x in t.rows(B * n))
    q, k = aoh_qk_rope(q, k, t.rope, **t.norms)
    aoh_kv_append_q8(k, v, LABELS, None, full, ring, SINK, WINDOW)
    t.lens = [n] * B
    for _ in range(3):
        q, k, v = (x.view(B, 1, -1, d) for x in t.rows(B))
        q, k = aoh_qk_rope(q, k, t.rope, start_pos=i32(t.lens), **t.norms)
        t.lens = [x + 1 for x in t.lens]
        lens = i32(t.lens)
        out = aoh_decode_step_q8(q[:, 0], k[:, 0], v[:, 0], full, ring, LABELS, lens, SINK, WINDOW)
        held = [torch.zeros((B, max(t.lens), HKV, d), dtype=BF, device=DEV) for _ in range(2)]
        aoh_kv_read_q8(full, ring, LABELS, None, lens, SINK, WINDOW, *held)
        want = attention.decode(f64(q[:, 0]), *map(f64, held), t.lens, LABELS, SINK, WINDOW)
        assert_parity(out.cpu(), want, BF, f"at {t.lens[0]}")
        assert (held[0][:, -1].float() - k[:, 0].float()).abs().max() <= k.float().abs().max() / 127
