"""The short convolution of few channels (csb_short_conv): its workgroups are whole wavefronts, and prompts of any lengths come out as the definition has them."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2005_05758_amd import short_conv
from test_gpu_scan import TYPES

pytestmark = pytest.mark.gpu

LAUNCHES = """
import json, os, sys, torch
from torch.profiler import ProfilerActivity, profile
from paper_2005_05758_amd import short_conv
x = {c: torch.randn(4096, c, device="cuda") for c in (1, 8, 9, 24, 33, 64, 65, 128, 129, 512)}
w = {c: torch.randn(c, 4, device="cuda") for c in x}
starts = [None] + [torch.arange(0, 4097, n, dtype=torch.int32, device="cuda") for n in (4, 32, 33, 64)]
starts[3] = torch.cat([starts[3], torch.tensor([4096], dtype=torch.int32, device="cuda")])
short_conv(x[8], w[8])
torch.cuda.synchronize()
with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
    for c in x:
        for s in starts:
            short_conv(x[c], w[c], starts=s)
    torch.cuda.synchronize()
p.export_chrome_trace(sys.argv[1])
"""


def test_workgroups_are_whole_wavefronts(tmp_path):
    """By a trace of the launches, in a process of its own."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    print("[conv] launches of 50 calls", flush=True)
    run = subprocess.run([sys.executable, "-c", LAUNCHES, str(tmp_path / "trace.json")], cwd=root, timeout=100, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert run.returncode == 0, run.stdout[-2000:]
    events = json.load(open(tmp_path / "trace.json"))["traceEvents"]
    threads = [int(np.prod(e["args"]["block"])) for e in events if e.get("cat") == "kernel" and "short_conv_kernel" in e["name"]]
    assert len(threads) == 50 and set(threads) <= {64, 128, 256}, threads


@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("C", [1, 3, 8, 16, 20, 64, 100])
@pytest.mark.parametrize("lengths", [[5000], [2047, 2048, 2049, 1, 0, 31], [33] * 120, [1] * 200 + [4200], [65, 0, 700, 32, 3]])
def test_prompts_of_few_channels(fmt, C, lengths):
    print(f"[conv] {fmt} {C} channels, lengths {lengths[:6]}", flush=True)
    t = torch.Generator().manual_seed(C + sum(lengths))
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    T, W = sum(lengths), 4
    x, w, b, S0 = rnd(T, C).to(TYPES[fmt]), 0.5 * rnd(C, W), rnd(C), rnd(len(lengths), W - 1, C).to(TYPES[fmt])
    at = np.concatenate([[0], np.cumsum(lengths)]).astype(int)
    want, off, state = ref.conv(*(ref.widen(v) for v in (x, w, b)), True, list(zip(at[:-1], at[1:])), list(range(len(lengths))), ref.widen(S0), fmt)
    S = S0.cuda()
    out = short_conv(x.cuda(), w.cuda(), b.cuda(), starts=torch.tensor(at, dtype=torch.int32, device="cuda"), state=S)
    torch.cuda.synchronize()
    assert ref.within(ref.widen(out), want, off, fmt) <= 0 and np.array_equal(ref.widen(S), state)
