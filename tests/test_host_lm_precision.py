"""The tolerances of tests/test_gpu_lm_precision.py tell 24 bits from 16: the model of the chunked delta rule is inside them with three
bfloat16 parts of every operand, and outside when any one of them has two.  So is the model of an adapter's second product."""
import numpy as np
import pytest

import lm_model as model
import lm_precision as cases


@pytest.mark.parametrize("fmt,DK", cases.HARDLY_DECAYING)
def test_every_operand_needs_its_third_part(fmt, DK):
    ins, S0, want, state = cases.hardly_decaying(fmt, DK)
    ins = [cases.widen(x) for x in ins]
    out, last = model.chunked(*ins, cases.SCALE, S0)
    assert cases.off(out, want) <= cases.KEEP / 4 and cases.off(last, state) <= cases.KEEP / 4
    for operand in model.OPERANDS:
        out, last = model.chunked(*ins, cases.SCALE, S0, {operand: 2})
        assert cases.off(out, want) > 1.5 * cases.KEEP, operand
        assert operand == "P" or cases.off(last, state) > 1.5 * cases.KEEP, operand


@pytest.mark.parametrize("fmt", sorted(cases.TYPES))
def test_outputs_that_cancel_need_p_s_third_part(fmt):
    ins = [cases.widen(x) for x in cases.cancelling()]
    want = cases.delta(*ins, 1.0, np.zeros((8, 64, 4)))[0][32:]
    for parts, right in ((3, True), (2, False)):
        out = model.chunked(*ins, 1.0, np.zeros((8, 64, 4)), {"P": parts})[0][32:]
        assert (np.abs(out - want) <= cases.CANCEL).all() == right


@pytest.mark.parametrize("fmt", sorted(cases.TYPES))
def test_the_adapters_sums_need_their_third_part(fmt):
    Y, X, A, B, want, allowed = cases.exact_adapter(fmt)
    t = A[0] @ X
    assert (np.float32(t) == t).all()                    # A X is exact in binary32
    for parts, right in ((3, True), (2, False)):
        assert (np.abs(Y + B[0] @ model.kept(t, parts) - want) <= allowed).all() == right
