"""Decodes over the 8-bit caches on given streams with the memory that the binding allocates for them: calls of two
streams run side by side while the current stream's tensors come and go."""
import pytest
import torch

from oracle import q8
from paper_2608_06849_amd import aoh_decode_q8, aoh_decode_step_q8
from tests.test_gpu_q8_decode import Run

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def stream_of(t):
    """Handle of the stream that a tensor's memory belongs to."""
    return [s["stream"] for s in torch.cuda.memory_snapshot()
            if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]


def test_two_streams_without_workspaces():
    runs = [Run(8, [0, 1, 0, 1], 128, 4, 60, lens, q8.E4M3, 80 + len(lens)) for lens in ([9000, 33], [700] * 70)]
    wants = [run.decode() for run in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for run, s in zip(runs, streams):
            got.append(aoh_decode_q8(run.q, run.full, run.ring, run.labels, run.lens, 4, 60, stream=s))
            # blocks of the workspaces' size on the current stream
            torch.full((32 << 20,), 255, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, wants[i % 2]), f"call {i}"
        assert stream_of(o) == [streams[i % 2].cuda_stream]


def test_step_on_a_stream_without_memory_of_its_own():
    run = Run(8, [0, 1], 64, 4, 60, [90, 33, 150], q8.I8, 90, tail=1)
    kn = torch.ones((3, 2, 64), dtype=BF, device=DEV)
    run.lens = run.lens + 1
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = aoh_decode_step_q8(run.q, kn, kn, run.full, run.ring, run.labels, run.lens, 4, 60, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    copy = got.clone()  # on the current stream, for which the block of `got` waits
    del got
    assert torch.equal(copy, run.decode())
