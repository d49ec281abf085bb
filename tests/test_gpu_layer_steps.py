"""Steps of the selective scan at their ends, with bounds that stay numbers behind a step of nothing.

layer_reference.scan takes what a step is off from what dt + bias is; of dt = -infinity that is 0 x infinity.  A step of dt = -2000 is zero too (e^-2000 is below binary64's
numbers), and its bound is zero: the reference is given that in place of -infinity."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref
import test_gpu_scan as scans
from paper_2005_05758_amd import selective_scan

pytestmark = pytest.mark.gpu


def extreme(fmt, T, channels, n, seed):
    """Inputs with steps that forget everything at once, of hardly anything, and of nothing at all; decays of zero among the others."""
    ins = scans.inputs(seed, T, channels, 1, n, fmt)
    x, dt, A = ins[:3]
    dt[20:25], dt[40:60], dt[61] = 300.0, -60.0, -math.inf
    dt[T // 2], dt[T - 3:T - 1, ::2] = 300.0, -math.inf
    A[:, 0] = 0.0
    return ins


def expected(ins, ranges, S0, fmt):
    wide = [ref.widen(v) for v in ins]
    wide[1] = np.where(np.isneginf(wide[1]), -2000.0, wide[1])
    x, dt, A, B, C, D, z, bias = wide
    want, off, S, S_off = ref.scan(x, dt, A, B, C, D, z, bias, True, ranges, list(range(len(ranges))), ref.widen(S0), fmt)
    assert np.isfinite(want).all() and np.isfinite(off).all() and np.isfinite(S).all() and np.isfinite(S_off).all()
    # the bounds ask for something: outputs and states of nothing, or of the last step's input alone, are outside of them almost everywhere
    assert (np.abs(want) > off + ref.HALF[fmt] * (np.abs(want) + off) + ref.TINY[fmt]).mean() > 0.98 and (np.abs(S) > S_off + ref.U * np.abs(S)).mean() > 0.98
    return want, off, S, S_off


@scans.types
@pytest.mark.parametrize("T,lengths", [(100, [100]), (800, [800]), (803, [700, 103]), (64, [1] * 64)])
@pytest.mark.parametrize("channels,n", [(20, 16), (64, 16), (20, 7)])
def test_steps_at_their_ends(fmt, T, lengths, channels, n):
    """In tiles, in chunks (whose decays multiply over such steps), and by the kernel for few tokens: outputs and states."""
    print(f"[steps] {fmt} lengths={lengths[:3]} {channels} channels, n = {n}", flush=True)
    ins = extreme(fmt, T, channels, n, seed=16)
    S0 = torch.randn(len(lengths), channels, n, generator=torch.Generator().manual_seed(17))
    at = [0] + np.cumsum(lengths).tolist()
    want, off, ws, ws_off = expected(ins, list(zip(at[:-1], at[1:])), S0, fmt)
    S = S0.cuda()
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in ins)
    out = selective_scan(x, dt, A, B, C, D=D, z=z, dt_bias=bias, starts=torch.tensor(at, dtype=torch.int32, device="cuda"), state=S)
    torch.cuda.synchronize()
    assert ref.within(ref.widen(out), want, off, fmt) <= 0 and ref.within(ref.widen(S), ws, ws_off, "f32") <= 0
