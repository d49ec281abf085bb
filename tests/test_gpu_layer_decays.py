"""Decays of the selective scan at their ends: -infinity (what -exp of a large number is) and numbers as large, which forget everything at a token's step."""
import math

import pytest
import torch

import test_gpu_scan as scans
from paper_2005_05758_amd import selective_scan

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# whole sequences in tiles, in chunks, and by the kernel for few tokens; a length of every rest by four
LENGTHS = {"tiles": [33, 34, 35, 36, 31, 1], "chunks": [700, 501, 0, 1, 402, 403], "few": [1, 2, 3, 4, 5, 0], "one": [1001]}


@pytest.mark.parametrize("A_low", [-math.inf, -3.0e38])
@pytest.mark.parametrize("n,channels", [(16, 64), (16, 70), (7, 24), (32, 64), (128, 20)])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_decays_that_forget_everything(fmt, lengths, n, channels, A_low):
    """As with a decay of -1e30, of which e^(s A) is zero too for these steps (0.001 and more): outputs and states are the same numbers."""
    lens = LENGTHS[lengths]
    T = sum(lens)
    print(f"[decays] {fmt} {lengths} {channels} channels, n = {n}, A = {A_low}", flush=True)
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in scans.inputs(T + n, T, channels, 1, n, fmt))
    bias = bias.clamp(min=-2.0)                          # s = ln(1 + e^(dt + bias)) with dt > -3: above 0.006
    S0 = torch.randn(len(lens), channels, n, device="cuda")
    starts = i32([0] + torch.tensor(lens).cumsum(0).tolist())
    got = []
    for low in (A_low, -1e30):
        A[:, ::3] = low
        S = S0.clone()
        got.append((selective_scan(x, dt, A, B, C, D=D, z=z, dt_bias=bias, starts=starts, state=S), S))
    torch.cuda.synchronize()
    (a, sa), (b, sb) = got
    assert bool(torch.isfinite(b).all()) and bool(torch.isfinite(sb).all())
    assert torch.equal(sa, sb) and torch.equal(a, b)


@pytest.mark.parametrize("A_low", [-math.inf, -float(torch.finfo(torch.float32).max), -3.0e38, -2.0e38])
@pytest.mark.parametrize("n,channels", [(16, 64), (7, 24)])
@pytest.mark.parametrize("lengths", sorted(LENGTHS))
def test_steps_of_zero_keep_the_state(lengths, n, channels, A_low):
    """Whatever the decay: e^(0 A) is one, and nothing comes in."""
    lens = LENGTHS[lengths]
    T = sum(lens)
    print(f"[decays] steps of zero, {lengths}, {channels} channels, n = {n}, A = {A_low}", flush=True)
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in scans.inputs(T + n, T, channels, 1, n, "f32"))
    S0 = torch.randn(len(lens), channels, n, device="cuda")
    starts = i32([0] + torch.tensor(lens).cumsum(0).tolist())
    A[:, ::2] = A_low
    S = S0.clone()
    out = selective_scan(x, torch.zeros_like(dt), A, B, C, softplus=False, starts=starts, state=S)
    seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
    want = (C.double() * S0.double()[seq]).sum(2)
    size = (C.double() * S0.double()[seq]).abs().sum(2)
    assert torch.equal(S, S0)
    assert bool(((out.double() - want).abs() <= (n + 3) * 2.0 ** -24 * size).all())       # a sum of n products, and its rounding


@pytest.mark.parametrize("T", [5, 130, 900])
def test_decays_that_are_not_numbers(T):
    """NaN spoils its channel and no other, whatever the steps are."""
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in scans.inputs(3, T, 24, 1, 16, "f32"))
    clean = selective_scan(x, dt, A, B, C, D=D, dt_bias=bias)
    A[5, 3] = math.nan
    got = selective_scan(x, dt, A, B, C, D=D, dt_bias=bias)
    rest = [c for c in range(24) if c != 5]
    assert torch.equal(got[:, rest], clean[:, rest]) and bool(torch.isnan(got[:, 5]).all())
