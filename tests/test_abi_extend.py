"""Refusals of the attention of new tokens: the C interface before anything is launched, and the binding for what the C
interface cannot see.  No GPU is needed."""
import pytest
import torch

import paper_2608_06849_amd as P
from paper_2608_06849_amd import aoh as A
from tests.test_abi_host import FAKE, _t

INV, UNS, WSP = A.AOH_ERR_INVALID_ARG, A.AOH_ERR_UNSUPPORTED, A.AOH_ERR_WORKSPACE
ALL = ("dense", "packed")


class Call:
    """Arguments of one call with good values for both entry points; a case changes some of them."""

    def __init__(self):
        self.q, self.k, self.v, self.out = _t((2, 5, 8, 128)), _t((2, 5, 2, 128)), _t((2, 5, 2, 128)), _t((2, 5, 8, 128))
        self.pq, self.pk, self.pv, self.pout = _t((9, 8, 128)), _t((9, 2, 128)), _t((9, 2, 128)), _t((9, 8, 128))
        self.start, self.cu, self.batch, self.max_new = FAKE, FAKE, 2, 7
        self.mask, self.n_sink, self.window, self.evict, self.append = b"\x00\x01", 4, 32, 0, 0
        self.full = A.AohPagedCache(FAKE, FAKE, FAKE, 8, 4, 1, 2, 0)
        self.ring = A.AohRingCache(FAKE, FAKE, 1, 36, 2)
        self.ws, self.ws_bytes = FAKE, 1 << 30

    def dense(self):
        return A.lib().aoh_extend(self.q, self.k, self.v, self.mask, self.start, self.full, self.ring, self.n_sink, self.window,
                                  self.evict, self.append, self.out, self.ws, self.ws_bytes, None)

    def packed(self):
        return A.lib().aoh_extend_varlen(self.pq, self.pk, self.pv, self.cu, self.batch, self.max_new, self.mask, self.start,
                                         self.full, self.ring, self.n_sink, self.window, self.evict, self.append, self.pout,
                                         self.ws, self.ws_bytes, None)


def put(**kw):
    return lambda c: [setattr(c, k, v) for k, v in kw.items()]


CASES = [
    (("dense",), put(q=None), INV, "q"), (("dense",), put(k=_t((2, 5, 2, 64)), v=_t((2, 5, 2, 64))), INV, "width"), (("dense",), put(v=_t((2, 5, 1, 128))), INV, "shapes"),
    (("dense",), put(k=_t((2, 6, 2, 128)), v=_t((2, 6, 2, 128))), INV, "tokens"), (("dense",), put(out=_t((2, 5, 4, 128))), INV, "out"),
    (("dense",), put(k=_t((2, 5, 2, 128), A.AOH_F32)), UNS, "k_new"),
    (("dense",), lambda c: [setattr(c, n, _t((2, 5, h, 128), A.AOH_F32)) for n, h in (("q", 8), ("k", 2), ("v", 2))], UNS, "out"),
    (("dense",), put(k=_t((2, 5, 3, 128)), v=_t((2, 5, 3, 128))), UNS, "multiple"),
    (("dense",), put(q=_t((2, 5, 34, 128)), out=_t((2, 5, 34, 128))), UNS, "16"),
    (("dense",), lambda c: [setattr(c, n, _t((2, 5, h, 96))) for n, h in (("q", 8), ("k", 2), ("v", 2), ("out", 8))], UNS, "D=96"),
    (("dense",), lambda c: [setattr(c, n, _t((1, 1 << 27, h, 128))) for n, h in (("q", 8), ("k", 2), ("v", 2), ("out", 8))], UNS, "many"),
    (("dense",), lambda c: [setattr(c, n, _t((1 << 16, 1 << 16, h, 128))) for n, h in (("q", 8), ("k", 2), ("v", 2), ("out", 8))], UNS, "many"),
    (ALL, put(evict=2), INV, "evict"), (ALL, put(append=-1), INV, "append"), (ALL, put(mask=None), INV, "head_is_streaming"),
    (ALL, put(mask=b"\x02\x00"), INV, "0/1"), (ALL, put(window=0), INV, "window"), (ALL, put(n_sink=-1), INV, "n_sink"),
    (ALL, put(full=None), INV, "kv_full"), (ALL, put(ring=None), INV, "kv_ring"), (ALL, put(window=33), INV, "capacity"),
    (ALL, lambda c: setattr(c.full, "n_seqs", 1), INV, "n_seqs"), (ALL, lambda c: setattr(c.ring, "batch", 1), INV, "batch"),
    (ALL, lambda c: setattr(c.full, "v_token_major", 1), UNS, "v_token_major"), (ALL, lambda c: setattr(c.full, "block_table", None), INV, "null"),
    (("packed",), put(cu=None), INV, "cu_seqlens"), (("packed",), put(batch=0), INV, "batch"), (("packed",), put(max_new=0), INV, "max_new"),
    (("packed",), put(pq=_t((2, 5, 8, 128))), INV, "dimensions"),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_refusals(n):
    names, change, status, text = CASES[n]
    for name in names:
        c = Call()
        change(c)
        st = getattr(c, name)()
        assert st == status and text in A.aoh_last_error(), (name, st, A.aoh_last_error())


def test_workspace_sizes():
    size = A.aoh_extend_workspace_bytes
    assert size(1, 1, 8, 2, 128) > 0 and size(1000, 100000, 32, 8, 64) > 0
    for bad in ((0, 1, 8, 2, 128), (1, 0, 8, 2, 128), (1, 1, 8, 0, 128), (1, 1, 7, 2, 128), (1, 1, 34, 2, 128), (1, 1, 8, 2, 96),
                (1, 1, 0, 2, 128)):
        assert size(*bad) == 0


def test_the_binding_refuses_what_the_library_cannot_see(monkeypatch):
    q, k = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64)
    full = P.PagedCache(torch.zeros(4, 1, 16, 64), torch.zeros(4, 1, 64, 16), torch.zeros(2, 2, dtype=torch.int32))
    ring = P.RingCache(torch.zeros(2, 1, 2, 16, 64), torch.zeros(2, 1, 2, 64, 16), 32)
    with pytest.raises(ValueError, match="cpu"):
        P.aoh_extend(q, k, k, [0, 1], None, full, ring, 4, 28)
    monkeypatch.setattr(A, "_on_gpu", lambda t, name: t.device)
    monkeypatch.setattr(A, "_q8_run", lambda *args: pytest.fail("not refused"))
    start = torch.zeros(2, dtype=torch.int32)
    for change, error, text in [
            (dict(q=q.half()), TypeError, "dtype"), (dict(k_new=k[..., :32]), ValueError, "width"),
            (dict(start_pos=start[:1]), ValueError, "start_pos"), (dict(start_pos=start.long()), ValueError, "start_pos"),
            (dict(head_is_streaming=[0]), ValueError, "labels"), (dict(out=torch.zeros(2, 3, 4, 32)), ValueError, "width"),
            (dict(workspace=torch.zeros(8, 8)[:, :4]), ValueError, "workspace"),
            (dict(kv_ring=P.RingCache(ring.k, ring.v, 33)), ValueError, "capacity"),
            (dict(kv_full=P.PagedCache(full.k.bfloat16(), full.v, full.block_table)), ValueError, "kv_full")]:
        args = dict(q=q, k_new=k, v_new=k, head_is_streaming=[0, 1], start_pos=start, kv_full=full, kv_ring=ring, n_sink=4, window=28)
        args.update(change)
        with pytest.raises(error, match=text):
            P.aoh_extend(**args)
    with pytest.raises(ValueError, match="cu_seqlens"):
        P.aoh_extend_varlen(q[0], k[0], k[0], torch.zeros(3, dtype=torch.long), 3, [0, 1], start, full, ring, 4, 28)
