"""Refusals of the norm and rotation calls: the C interface before anything is launched, and the binding for what the C
interface cannot see.  No GPU is needed."""
import ctypes

import pytest
import torch

import paper_2608_06849_amd as P
from paper_2608_06849_amd import aoh as A
from tests.test_abi_host import FAKE, _t

INV, UNS = A.AOH_ERR_INVALID_ARG, A.AOH_ERR_UNSUPPORTED
ALL = ("rope", "append", "packed")


class Call:
    """Arguments of one call with good values for every entry point; a case changes some of them."""

    def __init__(self):
        self.q, self.k, self.v = _t((2, 5, 8, 128)), _t((2, 5, 2, 128)), _t((2, 5, 2, 128))
        self.pq, self.pk, self.pv = _t((9, 8, 128)), _t((9, 2, 128)), _t((9, 2, 128))
        self.qo, self.ko, self.pqo = _t((2, 5, 8, 128)), _t((2, 5, 2, 128)), _t((9, 8, 128))
        self.q_norm = self.k_norm = None
        self.eps, self.pos, self.start, self.cu, self.batch, self.max_new = 1e-6, None, FAKE, FAKE, 2, 7
        self.rope = A.AohRope(FAKE, None, 64, 1, 0, 1.0)
        self.mask, self.n_sink, self.window = b"\x00\x01", 4, 32
        self.full = A.AohPagedCache(FAKE, FAKE, FAKE, 8, 4, 1, 2, 0)
        self.ringc = A.AohRingCache(FAKE, FAKE, 1, 36, 2)

    def axis(self, *axes, n_axes):
        self.keep = ctypes.create_string_buffer(bytes(axes), len(axes))
        self.rope.axis, self.rope.n_axes, self.rope.n_pairs = ctypes.cast(self.keep, ctypes.c_void_p), n_axes, len(axes)

    def rope_(self):
        return A.lib().aoh_qk_rope(self.q, self.k, self.q_norm, self.k_norm, self.eps, self.rope, self.pos, self.start,
                                   self.qo, self.ko, None)

    def append_(self):
        return A.lib().aoh_kv_append_rope(self.q, self.k, self.v, self.q_norm, self.k_norm, self.eps, self.rope, self.pos,
                                          self.mask, self.start, self.full, self.ringc, self.n_sink, self.window, self.qo,
                                          None)

    def packed_(self):
        return A.lib().aoh_kv_append_rope_varlen(self.pq, self.pk, self.pv, self.cu, self.batch, self.max_new, self.q_norm,
                                                 self.k_norm, self.eps, self.rope, self.pos, self.mask, self.start,
                                                 self.full, self.ringc, self.n_sink, self.window, self.pqo, None)


def put(**kw):
    return lambda c: [setattr(c, k, v) for k, v in kw.items()]


def rope(**kw):
    return lambda c: [setattr(c.rope, k, v) for k, v in kw.items()]


D = (_t, (128,))
CASES = [
    (ALL, rope(inv_freq=None), INV, "inv_freq"), (ALL, rope(n_pairs=0), INV, "n_pairs"), (ALL, rope(n_pairs=65), INV, "n_pairs"),
    (ALL, rope(n_axes=0), UNS, "n_axes"), (ALL, rope(n_axes=5), UNS, "n_axes"), (ALL, rope(interleaved=2), INV, "interleaved"),
    (ALL, rope(scale=float("nan")), INV, "scale"), (ALL, rope(n_axes=2), INV, "positions"), (ALL, rope(inv_freq=FAKE + 2), INV, "aligned"),
    (ALL, lambda c: c.axis(0, 1, 2, n_axes=2), INV, "axis[2]"), (ALL, put(eps=-1.0), INV, "eps"), (ALL, put(eps=float("nan")), INV, "eps"),
    (ALL, put(eps=float("inf")), INV, "eps"), (ALL, put(q_norm=_t((64,))), INV, "q_norm"), (ALL, put(k_norm=_t((128, 1))), INV, "k_norm"),
    (ALL, put(q_norm=_t((128,)), k_norm=_t((128,), A.AOH_F32)), INV, "dtypes"), (ALL, put(rope=None, pos=FAKE), INV, ""),
    (ALL, put(pos=FAKE + 1), INV, "aligned"),
    (("rope",), put(q=None, k=None, qo=None, ko=None), INV, "both null"), (("rope",), put(rope=None), INV, "neither"),
    (("rope",), put(qo=None), INV, "q_out"), (("rope",), put(k=None), INV, "k_out"), (("rope",), put(q=None, qo=None, q_norm=_t((128,))), INV, "norm"),
    (("rope",), put(qo=_t((2, 5, 4, 128))), INV, "shape"), (("rope",), put(qo=_t((2, 5, 8, 128), A.AOH_F32)), UNS, "q_out"),
    (("rope",), put(k=_t((2, 6, 2, 128)), ko=_t((2, 6, 2, 128))), INV, "tokens"), (("rope",), put(k=_t((2, 5, 2, 128), A.AOH_F32)), UNS, "k"),
    (("rope",), put(qo=_t((2, 5, 8, 128), stride=(10240, 2048, 128, 1))), INV, "in place"),
    (("rope",), put(q=_t((1 << 14, 1 << 14, 8, 128)), qo=_t((1 << 14, 1 << 14, 8, 128)), k=None, ko=None), UNS, "many"),
    (("rope",), put(q=_t((2, 5, 8, 96)), qo=_t((2, 5, 8, 96)), k=None, ko=None), UNS, "D=96"),
    (("append",), put(qo=None), INV, "q_out"), (("append",), put(q=None, qo=None, q_norm=_t((128,))), INV, "q_norm"),
    (("append",), put(v=_t((2, 5, 1, 128))), INV, "shapes"), (("append",), put(q=_t((2, 6, 8, 128)), qo=_t((2, 6, 8, 128))), INV, "tokens"),
    (("append",), put(k=None), INV, "k_new"), (("append", "packed"), put(mask=None), INV, "head_is_streaming"),
    (("append", "packed"), put(mask=b"\x00\x02"), INV, "0/1"), (("append", "packed"), put(full=None), INV, "kv_full"),
    (("append", "packed"), put(ringc=None), INV, "kv_ring"), (("append", "packed"), put(window=0), INV, "window"),
    (("append", "packed"), put(window=33), INV, "capacity"), (("append", "packed"), lambda c: setattr(c.full, "n_seqs", 1), INV, "n_seqs"),
    (("append", "packed"), lambda c: setattr(c.ringc, "batch", 1), INV, "batch"),
    (("append",), put(k=_t((1, 1 << 27, 2, 128)), v=_t((1, 1 << 27, 2, 128)), q=None, qo=None), UNS, "many"),
    (("packed",), put(cu=None), INV, "cu_seqlens"), (("packed",), put(batch=0), INV, "batch"), (("packed",), put(max_new=0), INV, "max_new"),
    (("packed",), put(pk=_t((2, 5, 2, 128))), INV, "dimensions"), (("packed",), put(pqo=_t((9, 4, 128))), INV, "shape"),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_refusals(n):
    names, change, status, text = CASES[n]
    for name in names:
        c = Call()
        change(c)
        st = getattr(c, name + "_")()
        assert st == status and text in A.aoh_last_error(), (name, st, A.aoh_last_error())


def test_rope_objects():
    f = torch.ones(8)
    with pytest.raises(ValueError):
        P.Rope(f.double())
    with pytest.raises(ValueError):
        P.Rope(f[::2])
    with pytest.raises(ValueError):
        P.Rope(f.view(2, 4))
    with pytest.raises(ValueError):
        P.Rope(f, axis=[0, 1])
    r = P.Rope(f, axis=[0, 1, 2, 0, 1, 2, 0, 1])
    assert r.n_axes == 3 and P.Rope(f).n_axes == 1
    with pytest.raises(AttributeError):
        r.inv_freq = f


def test_the_binding_refuses_what_the_library_cannot_see(monkeypatch):
    r = P.Rope(torch.ones(32))
    q, k = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64)
    with pytest.raises(ValueError, match="cpu"):
        P.aoh_qk_rope(q, k, r)
    with pytest.raises(ValueError, match="neither"):
        P.aoh_qk_rope(None, None, r)
    monkeypatch.setattr(A, "_on_gpu", lambda t, name: t.device)
    monkeypatch.setattr(A, "_q8_run", lambda *args: pytest.fail("not refused"))
    pos = torch.zeros(6, dtype=torch.int32)
    full = P.PagedCache(torch.zeros(4, 1, 16, 64), torch.zeros(4, 1, 64, 16), torch.zeros(2, 2, dtype=torch.int32))
    ring = P.RingCache(torch.zeros(2, 1, 2, 16, 64), torch.zeros(2, 1, 2, 64, 16), 32)

    def append(**kw):
        a = dict(q=q, k_new=k, v_new=k, rope=r, head_is_streaming=[0, 1], start_pos=None, kv_full=full, kv_ring=ring, n_sink=4,
                 window=28)
        a.update(kw)
        return P.aoh_kv_append_rope(**a)

    for call, error, text in [
            (lambda: P.aoh_qk_rope(q.half(), k, r), TypeError, "dtype"),
            (lambda: P.aoh_qk_rope(q, k[..., :32], r), ValueError, "width"),
            (lambda: P.aoh_qk_rope(q, k, r, positions=pos[:5]), ValueError, "positions"),
            (lambda: P.aoh_qk_rope(q, k, r, positions=pos.long()), ValueError, "positions"),
            (lambda: P.aoh_qk_rope(q, k, r, start_pos=pos[:1]), ValueError, "start_pos"),
            (lambda: P.aoh_qk_rope(q, k, r, q_norm=torch.ones(32)), ValueError, "q_norm"),
            (lambda: P.aoh_qk_rope(q, k, P.Rope(torch.ones(32, device="meta"))), ValueError, "rotation"),
            (lambda: append(head_is_streaming=[0, 1, 1]), ValueError, "labels"),
            (lambda: append(start_pos=pos[:1]), ValueError, "start_pos"),
            (lambda: append(kv_full=P.PagedCache(full.k.bfloat16(), full.v, full.block_table)), ValueError, "kv_full"),
            (lambda: append(kv_full=P.PagedCache(full.k, full.v, full.block_table.long())), ValueError, "block_table"),
            (lambda: append(kv_full=P.PagedCache(full.k[..., :32].contiguous(), full.v[:, :, :32].contiguous(), full.block_table)),
             ValueError, "width"),
            (lambda: append(kv_ring=P.RingCache(ring.k, ring.v, 33)), ValueError, "capacity"),
            (lambda: append(kv_ring=P.RingCache(torch.zeros(2, 2, 2, 16, 64)[:, :1], ring.v, 32)), ValueError, "contiguous"),
            (lambda: append(kv_ring=P.RingCache(ring.k, ring.v[:1], 32)), ValueError, "contiguous"),
    ]:
        with pytest.raises(error, match=text):
            call()
