"""Refusals of the 8-bit caches' entry points: the C interface rejects invalid arguments before anything is launched,
and the binding rejects tensors that the C interface cannot check.  No GPU is needed."""
import ctypes

import pytest
import torch

import paper_2608_06849_amd as P
from paper_2608_06849_amd import aoh as A
from tests.test_abi_host import FAKE, _t

INV, UNS, WSP = A.AOH_ERR_INVALID_ARG, A.AOH_ERR_UNSUPPORTED, A.AOH_ERR_WORKSPACE


def _caches(heads=1, seqs=2):
    full = A.AohPagedCacheQ8(FAKE, FAKE, FAKE, FAKE, 8, 4, heads, seqs, A.AOH_E4M3)
    ring = A.AohRingCacheQ8(FAKE, FAKE, FAKE, heads, 36, seqs, A.AOH_E4M3)
    return full, ring


class Call:
    """Arguments of one call with every entry point's good values; a case changes some of them."""

    def __init__(self):
        self.full, self.ring = _caches()
        self.k, self.v, self.pk, self.pv = _t((2, 5, 2, 128)), _t((2, 5, 2, 128)), _t((9, 2, 128)), _t((9, 2, 128))
        self.q, self.out, self.kn, self.vn = _t((2, 8, 128)), _t((2, 8, 128)), _t((2, 2, 128)), _t((2, 2, 128))
        self.mask, self.n_sink, self.window, self.pos, self.cu = b"\x00\x01", 4, 32, FAKE, FAKE
        self.batch, self.max_new, self.ws = 2, 7, FAKE
        self.ws_bytes = A.aoh_decode_q8_workspace_bytes(2, 8, 128)

    def append(self):
        return A.lib().aoh_kv_append_q8(self.k, self.v, self.mask, self.pos, self.full, self.ring, self.n_sink,
                                        self.window, None)

    def varlen(self):
        return A.lib().aoh_kv_append_q8_varlen(self.pk, self.pv, self.cu, self.batch, self.max_new, self.mask, self.pos,
                                               self.full, self.ring, self.n_sink, self.window, None)

    def read(self):
        return A.lib().aoh_kv_read_q8(self.full, self.ring, self.mask, None, self.pos, self.n_sink, self.window, self.k,
                                      self.v, None)

    def decode(self):
        return A.lib().aoh_decode_q8(self.q, self.full, self.ring, self.mask, self.pos, self.n_sink, self.window,
                                     self.out, self.ws, self.ws_bytes, None)

    def step(self):
        return A.lib().aoh_decode_step_q8(self.q, self.kn, self.vn, self.full, self.ring, self.mask, self.pos,
                                          self.n_sink, self.window, self.out, self.ws, self.ws_bytes, None)


ALL = ("append", "varlen", "read", "decode", "step")


def _refused(call, name, status, text):
    st = getattr(call, name)()
    assert st == status and text in A.aoh_last_error(), (name, st, A.aoh_last_error())


@pytest.mark.parametrize("name", ALL)
def test_common_refusals(name):
    def case(status, text, **change):
        c = Call()
        for path, value in change.items():
            obj, *field = path.split("__")
            if field:
                setattr(getattr(c, obj), field[0], value)
            else:
                setattr(c, obj, value)
        _refused(c, name, status, text)

    case(INV, "window", window=0)
    case(INV, "n_sink", n_sink=-1)
    case(UNS, "too large", n_sink=1 << 30, window=1 << 30)
    case(INV, "head_is_streaming", mask=None)
    case(INV, "0/1", mask=b"\x00\x02")
    case(INV, "kv_full", full__k=None)
    case(INV, "kv_full", full__scales=None)
    case(INV, "kv_ring", ring__scales=None)
    case(INV, "16-byte aligned", full__scales=FAKE + 8)
    case(INV, "16-byte aligned", ring__v=FAKE + 8)
    case(INV, "kv_full", full__block_table=None)
    case(INV, "empty cache", full__num_pages=0)
    case(INV, "n_seqs", full__n_seqs=1)
    case(INV, "kv_ring.batch", ring__batch=1)
    case(INV, "capacity", ring__capacity=37)
    case(UNS, "format 0", full__format=A.AOH_BF16)
    case(UNS, "format 9", ring__format=9)
    case(INV, "different formats", ring__format=A.AOH_I8)
    case(INV, "kv_ring is null", ring=None, **({"mask": b"\x01"} if name in ("decode", "step") else {}))
    case(INV, "no cache given" if name in ("decode", "step") else "kv_full is null", full=None,
         **({"ring": None} if name in ("decode", "step") else {}))


@pytest.mark.parametrize("name,shape,status,text", [
    ("append", (2, 5, 2, 96), UNS, "supported: 64, 128"),
    ("append", (2, 5, 0, 128), INV, "k_new"),
    ("append", (2, (1 << 26) + 1, 2, 128), UNS, "too many"),
    ("append", (2, 5, 70, 128), UNS, "Hkv"),
    ("read", (2, 5, 2, 32), UNS, "supported: 64, 128"),
    ("read", (0, 5, 2, 128), INV, "size 0"),
])
def test_row_tensors(name, shape, status, text):
    c = Call()
    c.k, c.v = _t(shape), _t(shape)
    _refused(c, name, status, text)


@pytest.mark.parametrize("name", ["append", "varlen", "read"])
def test_pairs_of_row_tensors(name):
    for a, b in (("k", "v"), ("pk", "pv")):
        if (a == "pk") != (name == "varlen"):
            continue
        c = Call()
        getattr(c, b).shape[0] -= 1
        _refused(c, name, INV, "shapes differ")
        c = Call()
        getattr(c, b).dtype = A.AOH_F32
        _refused(c, name, UNS, "dtype")
        for field, value in (("data", None), ("data", FAKE + 4)):
            c = Call()
            setattr(getattr(c, a), field, value)
            _refused(c, name, INV, "pointer")
        c = Call()
        getattr(c, a).stride[0] = 3
        _refused(c, name, INV, "stride")
    c = Call()
    c.k.dtype = c.v.dtype = c.pk.dtype = c.pv.dtype = A.AOH_E4M3
    _refused(c, name, UNS, "dtype")


def test_packed_counts():
    for change, text in ((dict(cu=None), "cu_seqlens"), (dict(batch=0), "batch"), (dict(max_new=0), "max_new")):
        c = Call()
        c.__dict__.update(change)
        _refused(c, "varlen", INV, text)


@pytest.mark.parametrize("name", ["decode", "step"])
def test_decode_refusals(name):
    def case(status, text, **change):
        c = Call()
        c.__dict__.update(change)
        _refused(c, name, status, text)

    case(INV, "lens", pos=None)
    case(UNS, "dtype", q=_t((2, 8, 128), A.AOH_F32))
    case(INV, "shape of q", out=_t((2, 4, 128)))
    case(UNS, "dtype", out=_t((2, 8, 128), 7))
    case(UNS, "supported: 64, 128", q=_t((2, 8, 32)), out=_t((2, 8, 32)))
    case(UNS, "multiple of Hkv", q=_t((2, 7, 128)), out=_t((2, 7, 128)))
    case(UNS, "> 16", q=_t((2, 34, 128)), out=_t((2, 34, 128)))
    case(WSP, "null", ws=None)
    case(WSP, "needed", ws_bytes=Call().ws_bytes - 1)
    case(INV, "aligned", ws=FAKE + 8)
    c = Call()
    c.full.max_pages_per_seq = 1 << 26   # 2 KV heads: 2^27 blocks a sequence
    assert c.full.max_pages_per_seq * 16 == 1 << 30
    c.full.n_heads, c.mask, c.q, c.out = 7, b"\x00" * 7 + b"\x01", _t((2, 8, 128)), _t((2, 8, 128))
    c.kn, c.vn = _t((2, 8, 128)), _t((2, 8, 128))
    _refused(c, name, UNS, "too many")


def test_step_refusals():
    for change, status, text in ((dict(kn=None), INV, "k_new"), (dict(vn=_t((2, 1, 128))), INV, "k_new / v_new"),
                                 (dict(kn=_t((2, 2, 128), A.AOH_F32)), UNS, "dtype"),
                                 (dict(kn=_t((2, 1, 2, 128))), INV, "dimensions")):
        c = Call()
        c.__dict__.update(change)
        _refused(c, "step", status, text)


def test_workspace_sizes():
    f = A.aoh_decode_q8_workspace_bytes
    assert f(0, 8, 128) == f(1, 0, 128) == f(1, 8, 96) == 0
    assert f(8, 32, 128) >= f(4, 32, 128) > 0 and f(100000, 32, 128) < 1 << 26


def test_cache_objects_check_their_tensors():
    table = torch.zeros((2, 4), dtype=torch.int32)
    for dt in (torch.float8_e4m3fn, torch.int8):
        full = P.PagedCacheQ8.allocate(8, 3, 64, dt, table, device="cpu")
        assert full.k.shape == (8, 3, 16, 64) and full.v.shape == (8, 3, 16, 4, 4, 4)
        assert full.scales.shape == (8, 3, 16, 2) and full.rows(1, 2)._desc.n_seqs == 1
        ring = P.RingCacheQ8.allocate(2, 1, 4, 33, 128, dt, device="cpu")
        assert ring.k.shape == (2, 1, 3, 16, 128) and ring._desc.capacity == 37
    k, v, s = full.k, full.v, full.scales
    with pytest.raises(TypeError):
        P.PagedCacheQ8(k.view(torch.uint8), v.view(torch.uint8), s, table)
    with pytest.raises(TypeError):
        P.PagedCacheQ8(k, v, s.view(torch.int8), table)
    for bad in ((k[:, :2], v, s, table), (k, v.flatten(2, 3), s, table), (k, v, s[:4], table),
                (k.transpose(0, 1).contiguous().transpose(0, 1), v, s, table), (k, v, s, table.long()),
                (k, v, s, table.flatten()), (k, v, s, table.t())):
        with pytest.raises(ValueError):
            P.PagedCacheQ8(*bad)
    with pytest.raises(ValueError):
        P.RingCacheQ8(ring.k, ring.v, ring.scales, 49)


def test_binding_refuses_host_tensors_and_mismatches():
    full = P.PagedCacheQ8.allocate(8, 1, 64, torch.int8, torch.zeros((2, 4), dtype=torch.int32), device="cpu")
    lens = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="caches are on cpu"):
        P.aoh_decode_q8(q, full, None, [0], lens, 0, 1)
    with pytest.raises(ValueError, match="no cache"):
        P.aoh_kv_append_q8(q, q, [0], lens, None, None, 0, 1)
    dev = torch.device("cuda", 0)
    with pytest.raises(ValueError, match="is on cpu"):
        A._q8_desc(q, "q", dev, 64)
    with pytest.raises(ValueError, match="width 128"):
        A._q8_desc(q, "q", torch.device("cpu"), 128)
    with pytest.raises(TypeError):
        A._q8_desc(q.half(), "q", torch.device("cpu"), 64)
    with pytest.raises(ValueError, match="int32"):
        A._q8_seqs(lens.long(), "lens", torch.device("cpu"), 2)
    with pytest.raises(ValueError, match="2 entries for 3"):
        A._q8_seqs(lens, "lens", torch.device("cpu"), 3)
    with pytest.raises(ValueError, match="labels"):
        A._q8_labels([0, 1], 3)


def test_cache_tensors_cannot_be_replaced():
    # the calls pass on the descriptor made with the object: another table or pool would not be seen
    full = A.PagedCacheQ8.allocate(3, 2, 64, torch.int8, torch.zeros(2, 2, dtype=torch.int32), device="cpu")
    ring = A.RingCacheQ8.allocate(2, 2, 4, 30, 64, torch.int8, device="cpu")
    for cache, names in ((full, ("k", "v", "scales", "block_table")), (ring, ("k", "v", "scales", "capacity"))):
        for name in names:
            with pytest.raises(AttributeError, match="cannot be replaced"):
                setattr(cache, name, getattr(cache, name))
