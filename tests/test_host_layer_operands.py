"""Refusals and workspace sizes of the operators around a recurrent layer, at the C entries: every call here is refused before anything is launched.
The addresses are numbers that nothing reads.  No GPU."""
import math

import pytest

from paper_2005_05758_amd.binding import VAL_BF16, VAL_F16, VAL_F32, csb_conv_args, csb_norm_args, csb_norm_operand, csb_scan_args, lib

EINVAL, EUNSUPPORTED = -1, -4
P = [4096 * (i + 1) for i in range(16)]                  # addresses

CONV = dict(type=VAL_BF16, channels=24, width=4, silu=1, n_seq=2, n_states=2, n_tokens=12, d_x=P[0], ldx=24, d_w=P[1], d_bias=P[2], d_state_in=P[3], d_state_out=P[3],
            d_out=P[4], ldo=24)
SCAN = dict(type=VAL_BF16, channels=16, groups=2, n=8, softplus=1, n_seq=2, n_tokens=40, d_x=P[0], d_dt=P[1], d_z=P[2], d_B=P[3], d_C=P[4], ldx=16, lddt=16, ldz=16, ldB=16,
            ldC=16, d_A=P[5], d_D=P[6], d_dt_bias=P[7], d_state_in=P[8], d_state_out=P[8], n_states=2, d_out=P[9], ldo=16)


def said(rc, name):
    assert lib().csb_last_error().decode().startswith(name + ": ")
    return rc


def conv(**change):
    return said(lib().csb_short_conv(csb_conv_args(**{**CONV, **change}), None), "csb_short_conv")


def scan(d_ws=None, **change):
    return said(lib().csb_selective_scan(csb_scan_args(**{**SCAN, **change}), d_ws, None), "csb_selective_scan")


def op(i, **kw):
    return csb_norm_operand(**{**dict(d=P[i], ld=16, type=VAL_F32, columns=0), **kw})


def norm(**change):
    good = dict(n_tokens=12, width=16, groups=1, after=1, before=1, scale=1.0, eps=1e-5, y=op(0), x=op(1), r=op(2), out=op(3))
    return said(lib().csb_block_norm(csb_norm_args(**{**good, **change}), None), "csb_block_norm")


NAMES = "type logits ld temperature top_k top_p min_p r n_rows vocab tokens probs ldprobs ws stream".split()


def sample(**change):
    good = dict(zip(NAMES, [VAL_F32, P[0], 64, P[1], P[2], P[3], P[4], P[5], 2, 64, P[6], P[7], 64, None, None]))
    return said(lib().csb_sample(*({**good, **change}[n] for n in NAMES)), "csb_sample")


@pytest.mark.parametrize("change", [dict(type=7), dict(type=-1), dict(channels=0), dict(width=0), dict(width=-1), dict(n_seq=-1), dict(n_seq=5), dict(n_tokens=-1),
                                    dict(ldx=23), dict(ldo=-24), dict(n_states=0), dict(d_w=None), dict(d_x=None), dict(d_out=None), dict(d_out=P[0]),
                                    dict(d_x=P[0] + 1), dict(d_w=P[1] + 2), dict(d_start=P[5] + 2), dict(d_state_out=P[3] + 1, type=VAL_F32)])
def test_short_conv(change):
    assert conv(**change) == EINVAL


def test_short_conv_of_more_than_it_takes():
    assert conv(width=9) == conv(n_tokens=1 << 31) == conv(n_tokens=0, n_seq=1 << 28) == EUNSUPPORTED
    assert conv(channels=(1 << 31) - 1, ldx=1 << 31, ldo=1 << 31, n_tokens=32 * (1 << 24), n_seq=1) == EUNSUPPORTED


@pytest.mark.parametrize("change", [dict(type=7), dict(channels=0), dict(channels=15), dict(groups=0), dict(groups=3), dict(n=0), dict(n_seq=-1), dict(n_seq=3),
                                    dict(n_tokens=-1), dict(ldx=15), dict(lddt=15), dict(ldz=15), dict(ldB=15), dict(ldC=15), dict(ldo=15), dict(n_states=0), dict(d_x=None), dict(d_dt=None),
                                    dict(d_A=None), dict(d_B=None), dict(d_C=None), dict(d_out=None), dict(d_dt=P[1] + 1), dict(d_A=P[5] + 2), dict(d_slot=P[10] + 1)])
def test_selective_scan(change):
    assert scan(**change) == EINVAL


@pytest.mark.parametrize("change", [dict(d_out=P[0], ldo=17), dict(d_out=P[1], lddt=17), dict(d_out=P[2], ldz=18), dict(d_out=P[3]), dict(d_out=P[4])])
def test_selective_scan_in_place_of_what_others_still_read(change):
    assert scan(**change) == EINVAL and b"out" in lib().csb_last_error()


def test_selective_scan_of_more_than_it_takes():
    assert scan(n=129, ldB=999, ldC=999) == scan(n_tokens=1 << 31) == scan(n_tokens=0, n_seq=1 << 28) == EUNSUPPORTED


def test_the_scans_workspace():
    size = lambda **change: lib().csb_scan_workspace_bytes(csb_scan_args(**{**SCAN, **change}))          # noqa: E731
    assert lib().csb_scan_workspace_bytes(None) == 0 and size(n_tokens=2) == size(n_tokens=40) == 0     # one launch
    long = dict(n_tokens=4096, n_seq=1)
    chunks = size(**long) // (16 * 8 * 4)
    assert 2 <= chunks <= 4096 // 32 + 1 + 128 and size(type=VAL_F32, **long) == size(**long)
    assert size(n_tokens=4096, n_seq=1, channels=65536) == 0                                             # enough workgroups without chunks
    assert scan(**long) == EINVAL and scan(d_ws=P[10] + 8, **long) == EINVAL
    for change in (dict(type=9), dict(n=129), dict(groups=3), dict(n_tokens=1 << 31), dict(n_seq=0), dict(n_seq=-1), dict(n_tokens=-1)):
        assert size(**{**long, **change}) == 0


NONE = csb_norm_operand()


@pytest.mark.parametrize("change", [dict(n_tokens=-1), dict(width=0), dict(groups=0), dict(groups=3), dict(after=3), dict(before=-1), dict(gate_kind=2), dict(eps=-1.0),
                                    dict(eps=math.nan), dict(eps=math.inf), dict(y=NONE, x=NONE), dict(y=NONE), dict(y=NONE, after=0, gate=op(5)), dict(out=NONE), dict(before=0, r=NONE),
                                    dict(out=op(2)), dict(y=op(0, ld=15)), dict(y=op(0, ld=11, columns=1)), dict(x=op(1, type=3)), dict(r=op(2, ld=-16)),
                                    dict(y=op(0, d=P[0] + 2)), dict(x=op(1, d=P[1] + 1, type=VAL_F16)), dict(d_after_w=P[5] + 2), dict(d_before_b=P[5] + 1)])
def test_block_norm(change):
    assert norm(**change) == EINVAL


@pytest.mark.parametrize("change", [dict(r=op(1, ld=17)), dict(r=op(1, type=VAL_BF16)), dict(r=op(1, columns=1)), dict(out=op(0, ld=32)), dict(out=op(0, type=VAL_F16)),
                                    dict(out=op(0, columns=1)), dict(gate=op(5), r=op(5, ld=20)), dict(y=op(0, columns=1), out=op(0))])
def test_block_norm_in_place_of_what_others_still_read(change):
    assert norm(**change) == EINVAL and b"input" in lib().csb_last_error()


def test_block_norm_of_more_than_it_takes():
    assert norm(groups=2) == norm(n_tokens=1 << 40) == EUNSUPPORTED
    wide = dict(y=op(0, ld=1 << 16), x=op(1, ld=1 << 16), r=op(2, ld=1 << 16), out=op(3, ld=1 << 16))
    assert norm(width=32769, **wide) == norm(width=1 << 16, groups=1, before=0, **wide) == EUNSUPPORTED


@pytest.mark.parametrize("change", [dict(type=9), dict(logits=None), dict(r=None), dict(tokens=None, probs=None), dict(ld=63), dict(ldprobs=63), dict(n_rows=-1), dict(vocab=0),
                                    dict(logits=P[0] + 2), dict(probs=P[7] + 1), dict(top_k=P[2] + 2), dict(tokens=P[6] + 1), dict(probs=P[0], ldprobs=65),
                                    dict(vocab=30000, ld=30000, ldprobs=30000), dict(vocab=30000, ld=30000, ldprobs=30000, ws=P[8] + 16)])
def test_sample(change):
    assert sample(**change) == EINVAL


def test_sample_of_more_than_it_takes():
    assert sample(vocab=(1 << 24) + 1, ld=1 << 25, ldprobs=1 << 25) == sample(n_rows=(1 << 21) + 1) == EUNSUPPORTED
    assert sample(n_rows=1 << 20, vocab=1 << 24, ld=1 << 24, ldprobs=1 << 24) == EUNSUPPORTED


def test_the_samples_workspace():
    size = lib().csb_sample_workspace_bytes
    assert size(0, 64000) == size(-1, 64000) == size(4, 24576) == size(4, 1) == 0
    assert 0 < size(1, 24577) < size(2, 24577) and size(2, 1 << 24) >= 2 * (1 << 24) // 16 * 4


def test_what_does_nothing():
    """No sequences, tokens or rows."""
    assert lib().csb_short_conv(csb_conv_args(**{**CONV, "n_seq": 0}), None) == 0
    assert lib().csb_selective_scan(csb_scan_args(**{**SCAN, "n_seq": 0}), None, None) == 0
    assert lib().csb_block_norm(csb_norm_args(n_tokens=0, width=16, groups=1, after=1, eps=1e-5), None) == 0
    assert lib().csb_sample(*dict(zip(NAMES, [0, None, 64, None, None, None, None, None, 0, 64, None, None, 0, None, None])).values()) == 0
    assert lib().csb_short_conv(None, None) == lib().csb_selective_scan(None, None, None) == lib().csb_block_norm(None, None) == EINVAL
