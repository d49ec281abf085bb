"""How many bits the operators of language models keep: inputs at which an operand with 16 bits in place of 24 is outside the
tolerance (tests/test_host_lm_precision.py shows that of each operand)."""
import sys

import numpy as np
import pytest
import torch

import lm_precision as cases
import lm_reference as ref
from lm_precision import HALF, TYPES, cancelling
from paper_2005_05758_amd import adapter_add, delta_chunked

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_outputs_that_cancel(fmt):
    """The weights of the output have 24 bits whatever its type: an output that is a small difference of two of them is as right as its
    type has it.  Each weight may be 3 units of 2^-24 off (the exponential 2, the sum's rounding 1), two of them 6; 8 are allowed.
    A weight of two bfloat16 parts is up to 32 units off."""
    ins = cancelling()
    say(f"[precision] outputs that cancel, {fmt}")
    want, _ = ref.delta(*(ref.widen(x) for x in ins), 1.0, [(0, ins[0].shape[0])], [-1], np.zeros((1, 8, 64, 4)))
    dev = [x.to(TYPES[fmt]).cuda() for x in ins[:3]] + [x.cuda() for x in ins[3:]]
    got = delta_chunked(*dev, scale=1.0)
    torch.cuda.synchronize()
    read = want[32:]
    assert 2.0 ** -13.5 < np.abs(read).min() and np.abs(read).max() < 2.0 ** -11.5
    off = np.abs(got.cpu().double().numpy()[32:] - read)
    assert (off <= 8 * 2.0 ** -24 + HALF[fmt] * np.abs(read) + 2.0 ** -25).all(), (off.max() * 2.0 ** 24, "units of 2^-24")


@pytest.mark.parametrize("fmt,DK", cases.HARDLY_DECAYING)
def test_states_keep_24_bits(fmt, DK):
    """Every operand between a chunk's products has 24 bits: states, and binary32 outputs, of chunks that hardly decay."""
    say(f"[precision] states, {fmt}, rows of {DK}")
    ins, S0, want, state = cases.hardly_decaying(fmt, DK)
    S = torch.from_numpy(S0[None]).float().cuda()
    got = delta_chunked(*(x.cuda() for x in ins), scale=cases.SCALE, state=S)
    torch.cuda.synchronize()
    assert cases.off(ref.widen(S)[0], state) <= cases.KEEP, cases.off(ref.widen(S)[0], state) / cases.KEEP
    far = np.abs(ref.widen(got) - want) - HALF[fmt] * np.abs(want)
    assert far.max() <= cases.KEEP * np.abs(want).max(), far.max() / np.abs(want).max() / cases.KEEP


@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_the_adapters_sums_keep_24_bits(fmt):
    """A X on its way to B: sums that need all of 24 bits."""
    say(f"[precision] adapter, {fmt}")
    Y, X, A, B, want, allowed = cases.exact_adapter(fmt)
    dev = [torch.from_numpy(x).to(TYPES[fmt]).cuda() for x in (X, A, B)]
    got = adapter_add(torch.from_numpy(Y).float().cuda(), *dev, torch.zeros(1, dtype=torch.int32, device="cuda"),
                      starts=torch.tensor([0, X.shape[1]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    off = np.abs(ref.widen(got) - want)
    assert (off <= allowed).all(), (off / allowed).max()
