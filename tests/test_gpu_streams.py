"""The calls that allocate a workspace themselves, on streams given to them: two streams side by side, no wait between
the calls, blocks of the current stream written meanwhile.  The results are those of the current stream."""
import pytest
import torch

from paper_2608_06849_amd import aoh_classify, aoh_decode_anchor, aoh_decode_reuse, aoh_head_mapping, aoh_kv_append
from tests.test_gpu_h2share import BF, DEV, _decode_setup

pytestmark = pytest.mark.gpu


def _weights(n, dm, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn((n, dm), device=DEV, generator=g) * 0.05).to(BF)


def _sets(name, seed):
    """A call of the entry point on a stream (None: the current one), with everything but its memory prepared."""
    if name == "classify":
        wq, wk = _weights(3 * 8 * 64, 256, seed).view(3, -1, 256), _weights(3 * 2 * 64, 256, seed + 1).view(3, -1, 256)
        return lambda s: aoh_classify(wq, wk, 64, 1, stream=s)
    if name == "mapping":
        w = [_weights(n * 64, 256, seed + n) for n in (8, 2)] * 2
        return lambda s: aoh_head_mapping(*w, 64, [0, 1], [1, 0], stream=s)
    k, v, full, ring = _decode_setup(2, 300, 8, 2, 64, [0, 1], 4, 60, seed)
    aoh_kv_append(k.to(DEV), v.to(DEV), [0, 1], torch.zeros(2, dtype=torch.int32, device=DEV), full, ring, 4, 60)
    lens = torch.tensor([300, 170], dtype=torch.int32, device=DEV)
    q = _weights(2 * 8, 64, seed).view(2, 8, 64)
    if name == "anchor":
        return lambda s: aoh_decode_anchor(q, full, ring, [0, 1], lens, 4, 60, 32, stream=s)
    lists = aoh_decode_anchor(q, full, ring, [0, 1], lens, 4, 60, 32)[1]
    return lambda s: (aoh_decode_reuse(q, full, ring, [0, 1], lens, 4, 60, lists, [0, -1], stream=s),)


@pytest.mark.parametrize("name", ["anchor", "reuse", "mapping", "classify"])
def test_two_streams_without_workspaces(name):
    calls = [_sets(name, seed) for seed in (100, 200)]
    wants = [call(None) for call in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for call, s in zip(calls, streams):
            got.append(call(s))
            torch.full((4 << 20,), 255, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for x, want in zip(r, wants[i % 2]):
            assert torch.equal(x, want), f"call {i}"
