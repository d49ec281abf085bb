"""The operators around a recurrent layer on another stream than the current one, with nothing that waits on the host (as test_gpu_streams.py, whose
tests these are): the blocks of a call's workspace and results are not in use by anybody else before and after it."""
import pytest
import torch

import test_gpu_streams as streams
from paper_2005_05758_amd import block_norm, sample, selective_scan, short_conv

pytestmark = pytest.mark.gpu
normal = streams.normal


def scan_inputs(seed, T=4000, C=256, n=16):
    return (normal(seed, T, C).bfloat16().cuda(), normal(seed + 1, T, C).bfloat16().cuda(), -normal(seed + 2, C, n).abs().cuda(),
            normal(seed + 3, T, 1, n).bfloat16().cuda(), normal(seed + 4, T, 1, n).bfloat16().cuda())


CALLS = {
    "short_conv": (lambda seed: (normal(seed, 3000, 512).bfloat16().cuda(), normal(seed + 1, 512, 4).cuda()), lambda ins, **kw: short_conv(*ins, **kw)),
    "selective_scan": (scan_inputs, lambda ins, **kw: selective_scan(*ins, **kw)),
    "block_norm": (lambda seed: (normal(seed, 700, 1024).cuda(), normal(seed + 1, 700, 1024).cuda()),
                   lambda ins, **kw: block_norm(ins[0], x=ins[1], after="rms", before="rms", **kw)),
    "sample": (lambda seed: (3 * normal(seed, 20, 70000).cuda(), normal(seed + 1, 20).abs().clamp(max=0.99).cuda(), torch.full((20,), 50, dtype=torch.int32, device="cuda")),
               lambda ins, **kw: sample(ins[0], ins[1], top_k=ins[2], probs=True, **kw)),
}


@pytest.fixture(autouse=True)
def these_calls(monkeypatch):
    monkeypatch.setattr(streams, "CALLS", CALLS)


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("test", ["test_the_workspace_is_nobody_elses_until_the_call_has_run", "test_results_do_not_lie_in_what_the_current_stream_still_writes",
                                  "test_results_stay_until_the_callers_stream_has_read_them"])
def test_another_stream(test, name):
    getattr(streams, test)(name)


def test_two_graphs_and_eager_calls_between():
    """Two captured calls and eager ones with workspaces of their own, replayed in turn."""
    for name in ("selective_scan", "sample"):
        make, call = CALLS[name]
        ins, other = make(1), make(2)
        want = [t.clone() for t in streams.results(call(ins))], [t.clone() for t in streams.results(call(other))]
        torch.cuda.synchronize()
        graphs, held = [], []
        for i in (ins, other):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                held.append(streams.results(call(i)))
            graphs.append(g)
        for _ in range(3):
            for g in graphs:
                g.replay()
                call(make(3))
            torch.cuda.synchronize()
            for h, w in zip(held, want):
                assert all(torch.equal(x, y) for x, y in zip(h, w))
