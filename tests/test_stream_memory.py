"""Memory that the binding allocates for a call belongs to the stream of the call: a block of another stream may be
given to that stream's next tensor while the call's kernels still use it.  The library and the streams are stand-ins, so
nothing runs and no GPU is needed."""
import contextlib
import types

import pytest
import torch

from paper_2608_06849_amd import aoh as A

BF = torch.bfloat16
B, HQ, HKV, D = 2, 4, 2, 64


class Library:
    """Every entry point returns 0; the 8-bit caches' ones are found under `packed` too."""

    def __init__(self):
        self.packed = self

    def __getattr__(self, name):
        return lambda *args: 0

    def __getitem__(self, name):
        return lambda *args: 0


@pytest.fixture
def trace(monkeypatch):
    """What was allocated on which stream, and for which other stream its end of life waits."""
    device = torch.device("cpu")
    home = types.SimpleNamespace(device=device, cuda_stream=0, name="current")
    t = types.SimpleNamespace(now=home, home=home, side=types.SimpleNamespace(device=device, cuda_stream=64, name="side"),
                              made=[], kept=[])

    @contextlib.contextmanager
    def on(stream):
        before, t.now = t.now, stream
        yield
        t.now = before

    def watched(make):
        def call(*args, **kw):
            x = make(*args, **kw)
            t.made.append((t.now, x))
            return x
        return call

    monkeypatch.setattr(A, "lib", Library)
    monkeypatch.setattr(A, "_q8_caches", lambda full, ring: (device, D, None, None))
    monkeypatch.setattr(A, "_q8_labels", lambda labels, n: bytes(labels))
    monkeypatch.setattr(A, "_current_stream", lambda index: 0)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: t.now)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    monkeypatch.setattr(torch, "empty_like", watched(torch.empty_like))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda x, s: t.kept.append((s, x)))
    return t


def rows(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


WQ, WK = rows(HQ * D, 128), rows(HKV * D, 128)
PROMPT, KV = rows(1, 5, HQ, D), rows(1, 5, HKV, D)
CU = torch.tensor([0, 5], dtype=torch.int32)
LENS = torch.ones(B, dtype=torch.int32)
Q, NEW = rows(B, HQ, D), rows(B, HKV, D)
CALLS = {
    "aoh_decode_q8": lambda **kw: A.aoh_decode_q8(Q, None, None, [0, 1], LENS, 4, 28, **kw),
    "aoh_decode_step_q8": lambda **kw: A.aoh_decode_step_q8(Q, NEW, NEW, None, None, [0, 1], LENS, 4, 28, **kw),
    "aoh_prefill": lambda **kw: A.aoh_prefill(PROMPT, KV, KV, [0, 1], 4, 28, **kw),
    "aoh_prefill_chunked": lambda **kw: A.aoh_prefill_chunked(PROMPT, KV, KV, [0, 1], 4, 28, 32, **kw),
    "aoh_prefill_append": lambda **kw: A.aoh_prefill_append(PROMPT, KV, KV, [0, 1], 4, 28, None, None, **kw),
    "aoh_prefill_varlen": lambda **kw: A.aoh_prefill_varlen(PROMPT[0], KV[0], KV[0], CU, 5, [0, 1], 4, 28, **kw),
    "aoh_decode": lambda **kw: A.aoh_decode(Q, None, None, [0, 1], LENS, 4, 28, **kw),
    "aoh_decode_step": lambda **kw: A.aoh_decode_step(Q, NEW, NEW, None, None, [0, 1], LENS, 4, 28, **kw),
    "aoh_decode_step_noalloc": lambda **kw: A.aoh_decode_step_noalloc(Q, NEW, NEW, None, None, [0, 1], LENS, 4, 28, **kw),
    "aoh_classify": lambda **kw: A.aoh_classify(WQ[None], WK[None], D, 1, **kw),
    "aoh_head_mapping": lambda **kw: A.aoh_head_mapping(WQ, WK, WQ, WK, D, [0, 1], [0, 1], **kw),
    "aoh_decode_anchor": lambda **kw: A.aoh_decode_anchor(Q, None, None, [0, 1], LENS, 4, 28, 8, **kw),
    "aoh_decode_reuse": lambda **kw: A.aoh_decode_reuse(Q, None, None, [0, 1], LENS, 4, 28, rows(B, 1, 8, dtype=torch.int32),
                                                        [0, 0], **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_is_its_streams(name, trace):
    result = CALLS[name](stream=trace.side)
    result = result if isinstance(result, tuple) else (result,)
    assert trace.made and all(s is trace.side for s, _ in trace.made), [s.name for s, _ in trace.made]
    # the caller may use results on its own stream: their memory waits for that one too
    assert [id(x) for s, x in trace.kept if s is trace.home] == [id(x) for x in result]
    assert trace.now is trace.home


@pytest.mark.parametrize("name", CALLS)
def test_without_a_stream_it_is_the_current_ones(name, trace):
    CALLS[name]()
    assert trace.made and all(s is trace.home for s, _ in trace.made) and not trace.kept
