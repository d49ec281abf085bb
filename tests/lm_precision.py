"""Cases that show how many bits an operator of language models keeps, with what they are allowed (test infrastructure)."""

import numpy as np
import torch

import lm_reference as ref
from lm_reference import widen                           # noqa: F401  (for the tests of these cases)

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit in the last place, of the value

# States and binary32 outputs: 8 units of 2^-24 of the largest entry.  A chunk's operands and sums are rounded to 24 bits a handful of times, each up to
# a unit of numbers no larger than that entry, independent of each other; later chunks make no earlier error larger.
KEEP = 2.0 ** -21
SCALE = 0.125
HARDLY_DECAYING = [("bf16", 64), ("bf16", 256), ("f16", 64), ("f16", 128), ("f16", 256), ("bf16", 128), ("f32", 64), ("f32", 128)]


def delta(q, k, v, g, beta, scale, S):
    """One sequence in 64 bits; S [heads_v, dk, dv].  Returns (out, S)."""
    out, state = ref.delta(q, k, v, g, beta, scale, [(0, v.shape[0])], [0], S[None])
    return out, state[0]


def off(got, want):
    return np.abs(got - want).max() / max(1e-30, np.abs(want).max())


def hardly_decaying(fmt, DK, T=190, HK=2, HV=4, DV=48):
    """Three chunks through which what is in the state stays there: (inputs, state before, outputs, state behind)."""
    t = torch.Generator().manual_seed(60 + DK)
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, generator=t), dim=-1).to(TYPES[fmt])   # noqa: E731
    ins = [unit(T, HK, DK), unit(T, HK, DK), torch.randn(T, HV, DV, generator=t).to(TYPES[fmt]), -0.02 * torch.rand(T, HV, generator=t) ** 3,
           torch.sigmoid(torch.randn(T, HV, generator=t))]
    S0 = widen(torch.randn(HV, DK, DV, generator=t))
    return (ins, S0, *delta(*(widen(x) for x in ins), SCALE, S0))


# Outputs that are small differences of two weights near 1: each weight may be 3 units of 2^-24 off (the exponential 2, the sum's rounding 1), two
# of them 6; 8 are allowed.  A weight of two bfloat16 parts is up to 32 units off.
CANCEL = 8 * 2.0 ** -24


def cancelling(seed=40, heads=8, dk=64, dv=4, pairs=16):
    """Pairs of tokens with keys of their own that write 1 and -1 hardly decayed from one to the other, then tokens that read the sum of
    a pair: two weights near 1 whose difference, some 2^-13, is the output.  Every number but the decays is exact in all types."""
    t = torch.Generator().manual_seed(seed)
    T = 3 * pairs
    q, k = torch.zeros(T, 1, dk), torch.zeros(T, 1, dk)
    v, beta = torch.zeros(T, heads, dv), torch.zeros(T, heads)
    g = -2.0 ** -13 * (1 + torch.rand(T, heads, generator=t))
    for j in range(pairs):
        k[2 * j, 0, 2 * j] = k[2 * j + 1, 0, 2 * j + 1] = 1.0
        v[2 * j], v[2 * j + 1] = 1.0, -1.0
        beta[2 * j] = beta[2 * j + 1] = 1.0
        g[2 * j] = -0.04 * torch.rand(heads, generator=t)
        q[2 * pairs + j, 0, 2 * j] = q[2 * pairs + j, 0, 2 * j + 1] = 1.0
        k[2 * pairs + j, 0, dk - 1] = 1.0
    return q, k, v, g, beta


def exact_adapter(fmt, rows=70, cols=96, batch=40, rank=8):
    """An adapter whose A X is exact in binary32 and needs all of its 24 bits: numbers of 8 bits at three places of a row, which X's three powers of two
    put side by side (binary16, of 5 bits of exponent: 2^-8, 1 and 2^8).  Returns (Y, X, A, B, the result, what it may be off): float64, values of the type.
    Only the second product and its sum with Y round: rank + 4 units of 2^-24 of the absolute values' sum."""
    g = np.random.default_rng(61)
    A, X = np.zeros((1, rank, cols)), np.zeros((cols, batch))
    A[0][:, [3, 40, 90]] = g.integers(129, 256, (rank, 3)) * g.choice([-1, 1], (rank, 1))
    X[3], X[40], X[90] = 2.0 ** 8, 1.0, 2.0 ** -8
    X *= g.choice([-1.0, 1.0], batch)
    B = widen(torch.from_numpy(g.normal(0, 1, (1, rows, rank))).to(TYPES[fmt]))
    Y = widen(torch.from_numpy(g.normal(0, 1, (rows, batch))).float())
    t = A[0] @ X
    return Y, X, A, B, Y + B[0] @ t, (rank + 4) * 2.0 ** -24 * (np.abs(Y) + np.abs(B[0]) @ np.abs(t))
