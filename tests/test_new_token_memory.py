"""Memory that norms and positions, their appends and running prompts allocate belongs to the stream of the call, as
tests/test_stream_memory.py has it for the other calls, whose stand-ins serve here too."""
import pytest
import torch

from paper_2608_06849_amd import aoh as A
from tests.test_stream_memory import BF, CU, D, HKV, HQ, KV, PROMPT, trace  # noqa: F401  (a fixture)


@pytest.fixture
def on_cpu(monkeypatch):
    monkeypatch.setattr(A, "_on_gpu", lambda t, name: t.device)


ROPE = A.Rope(torch.ones(D // 2))
TABLE = torch.zeros((1, 4), dtype=torch.int32)
FULL = A.PagedCache.allocate(4, 1, D, BF, TABLE, device="cpu")
RING = A.RingCache.allocate(1, 1, 4, 28, D, BF, device="cpu")
CALLS = {
    "aoh_qk_rope": lambda **kw: A.aoh_qk_rope(PROMPT, KV, ROPE, **kw),
    "aoh_kv_append_rope": lambda **kw: A.aoh_kv_append_rope(PROMPT, KV, KV, ROPE, [0, 1], None, FULL, RING, 4, 28, **kw),
    "aoh_kv_append_rope_varlen": lambda **kw: A.aoh_kv_append_rope_varlen(PROMPT[0], KV[0], KV[0], CU, 5, ROPE, [0, 1], None,
                                                                          FULL, RING, 4, 28, **kw),
    "aoh_extend": lambda **kw: A.aoh_extend(PROMPT, KV, KV, [0, 1], None, FULL, RING, 4, 28, **kw),
    "aoh_extend_varlen": lambda **kw: A.aoh_extend_varlen(PROMPT[0], KV[0], KV[0], CU, 5, [0, 1], None, FULL, RING, 4, 28, **kw),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_is_its_streams(name, trace, on_cpu):  # noqa: F811
    result = CALLS[name](stream=trace.side)
    result = result if isinstance(result, tuple) else (result,)
    assert trace.made and all(s is trace.side for s, _ in trace.made), [s.name for s, _ in trace.made]
    assert [id(x) for s, x in trace.kept if s is trace.home] == [id(x) for x in result]
    assert trace.now is trace.home


@pytest.mark.parametrize("name", CALLS)
def test_without_a_stream_it_is_the_current_ones(name, trace, on_cpu):  # noqa: F811
    CALLS[name]()
    assert trace.made and all(s is trace.home for s, _ in trace.made) and not trace.kept
