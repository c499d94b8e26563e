"""Packed prompts attended to and written into 8-bit caches that held nothing before, then captured steps: every byte
that the steps read has to come from the calls under test."""
import pytest
import torch

import synth
from oracle import q8
from paper_2608_06849_amd import aoh_decode_q8_workspace_bytes, aoh_decode_step_q8, aoh_kv_append_q8_varlen, aoh_prefill_varlen
from tests.test_gpu_q8_cache import int32
from tests.test_gpu_q8_decode import Run

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", [q8.E4M3, q8.I8])
def test_steps_read_what_the_prompts_wrote(fmt, d):
    hq, labels, n_sink, window, steps = 8, [1, 0], 16, 112, 4
    lens = [37, 260, 16]
    run = Run(hq, labels, d, n_sink, window, lens, fmt, 130 + d, tail=steps)
    for c in (run.full, run.ring):  # NaN codes, as K and V, and infinite scales
        c.k.view(torch.uint8).fill_(0x7F)
        c.v.view(torch.uint8).fill_(0xFF)
        c.scales.fill_(255)
    k, v = (torch.cat([x[i, :n] for i, n in enumerate(lens)]).to(DEV) for x in (run.k, run.v))
    q = torch.from_numpy(synth.gaussian((sum(lens), hq, d), 131, "q8-serve").astype("float32")).to(BF).to(DEV)
    cu = int32([0, 37, 297, 313])
    prompt = aoh_prefill_varlen(q, k, v, cu, max(lens), labels, n_sink, window)
    aoh_kv_append_q8_varlen(k, v, cu, max(lens), labels, None, run.full, run.ring, n_sink, window)
    assert torch.isfinite(prompt).all()
    run.check(run.decode(), what="after the prompts")
    kn, vn = (torch.zeros((3, 2, d), dtype=BF, device=DEV) for _ in range(2))
    ws = torch.empty(aoh_decode_q8_workspace_bytes(3, hq, d), dtype=torch.uint8, device=DEV)
    out, now = torch.zeros_like(run.q), run.lens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        now += 1
        aoh_decode_step_q8(run.q, kn, vn, run.full, run.ring, labels, now, n_sink, window, out=out, workspace=ws)
    now.copy_(run.lens)
    for s in range(steps):
        for i, n in enumerate(lens):
            kn[i], vn[i] = run.k[i, n + s].to(DEV), run.v[i, n + s].to(DEV)
        graph.replay()
        run.check(out, [n + s + 1 for n in lens], f"step {s}")
