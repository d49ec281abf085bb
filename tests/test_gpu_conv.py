"""The short causal convolution (csb_short_conv) against its definition in 64 bits on the host."""
import math
import sys

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2005_05758_amd import short_conv
from paper_2005_05758_amd.binding import CsbError, csb_conv_args, lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
types = pytest.mark.parametrize("fmt", sorted(TYPES))


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if x is not None else None


def inputs(seed, T, C, W, fmt):
    t = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    return rnd(T, C).to(TYPES[fmt]), rnd(C, W), rnd(C)


def check(fmt, T, C, W, lengths=None, lens=None, slots=None, n_states=None, seed=0, silu=True, bias=True, state=True, keep=True, place=None, change=None):
    say(f"[conv] {fmt} T={T} C={C} W={W} lengths={lengths} lens={lens} slots={slots} {place or ''}")
    x, w, b = inputs(seed, T, C, W, fmt)
    if not bias:
        b = None
    if change:
        change(x)
    N = len(lengths) if lengths is not None else 1
    first = np.concatenate([[0], np.cumsum(lengths)]).astype(int) if lengths is not None else np.array([0, T])
    ranges = [(first[i], first[i] + min(max(lens[i], 0), first[i + 1] - first[i]) if lens is not None else first[i + 1]) for i in range(N)]
    n_states = n_states or N
    S0 = torch.randn(n_states, W - 1, C, generator=torch.Generator().manual_seed(seed + 1)).to(TYPES[fmt])
    where = [s if 0 <= s < n_states else -1 for s in slots] if slots is not None else list(range(N))
    with np.errstate(invalid="ignore"):
        want, off, ws = ref.conv(ref.widen(x), ref.widen(w), ref.widen(b) if bias else np.zeros(C), silu, ranges, where if state else [-1] * N, ref.widen(S0), fmt)
    xd = place(x) if place else x.cuda()
    S = S0.cuda() if state else None
    out = torch.full((T, C), 7.0, dtype=TYPES[fmt], device="cuda")
    got = short_conv(xd, w.cuda(), b.cuda() if bias else None, silu=silu, starts=i32([int(f) for f in first]) if lengths is not None else None, lens=i32(lens),
                     slots=i32(slots), state=S, out=out, **({} if keep else {"state_out": None}))
    torch.cuda.synchronize()
    assert got is out
    o = ref.widen(out)
    there = ~np.isnan(want)
    if change is None:
        assert (o[~there] == 7.0).all(), "tokens that no sequence takes are not written"
        assert ref.within(o, want, off, fmt) <= 0
        if state:
            assert np.array_equal(ref.widen(S), ws if keep else ref.widen(S0))
    return o, want, off


@types
@pytest.mark.parametrize("T,C,W", [(1, 1, 1), (1, 8, 4), (2, 3, 3), (3, 64, 4), (16, 9, 2), (17, 513, 4), (64, 65, 8), (65, 130, 5), (200, 520, 4), (131, 40, 6), (67, 30, 7)])
def test_one_sequence(fmt, T, C, W):
    check(fmt, T, C, W, seed=T + C)


@types
def test_packed_sequences(fmt):
    lengths = [1, 0, 64, 3, 128, 65, 0, 0, 31, 2, 300]
    check(fmt, sum(lengths), 48, 4, lengths=lengths, seed=3)
    check(fmt, sum(lengths) + 5, 21, 4, lengths=lengths, slots=[11, 3, -1, 0, 99, 7, 5, 2, 1, -2, 8], n_states=12, seed=4)
    check(fmt, sum(lengths), 20, 3, lengths=lengths, lens=[1, 0, 63, -4, 65, 99, 2, 0, 0, 1, 40], seed=5)


@types
@pytest.mark.parametrize("W", [2, 4, 8])
def test_sequences_shorter_than_the_state(fmt, W):
    """A state keeps what the tokens have not pushed out."""
    check(fmt, 28, 24, W, lengths=[0, 1, 2, 3, 4, 5, 6, 7], slots=[7, 6, 5, 4, 3, 2, 1, 0], seed=6)


def test_many_sequences():
    g = np.random.default_rng(1)
    lengths = [int(v) for v in g.integers(0, 5, 700)]
    check("bf16", sum(lengths), 16, 4, lengths=lengths, slots=[int(v) for v in g.permutation(700)], seed=6)


def test_forms():
    check("f32", 90, 33, 4, lengths=[70, 20], seed=7, state=False)
    check("f16", 90, 33, 4, lengths=[70, 20], seed=8, keep=False)
    check("bf16", 90, 33, 4, lengths=[70, 20], seed=8, silu=False)
    check("bf16", 90, 33, 4, lengths=[70, 20], seed=8, bias=False)


@types
def test_state_into_another_buffer(fmt):
    """The last inputs go to a second buffer; a sequence of no tokens takes its state over as it is."""
    x, w, b = (v.cuda() for v in inputs(9, 80, 24, 4, fmt))
    S = torch.randn(3, 3, 24, device="cuda").to(TYPES[fmt])
    into, starts, keep = torch.full_like(S, 5.0), i32([0, 70, 70, 80]), S.clone()
    a = short_conv(x, w, b, starts=starts, state=S, state_out=into)
    assert torch.equal(S, keep)
    c = short_conv(x, w, b, starts=starts, state=S)
    torch.cuda.synchronize()
    assert torch.equal(a, c) and torch.equal(into, S) and torch.equal(into[1], keep[1]) and not torch.equal(into[0], keep[0])


@types
def test_in_parts(fmt):
    """A prompt in parts, each from the state of the one before, and token by token: the same bits."""
    x, w, b = (v.cuda() for v in inputs(10, 150, 40, 4, fmt))
    S, P = (torch.zeros(1, 3, 40, dtype=TYPES[fmt], device="cuda") for _ in range(2))
    whole = short_conv(x, w, b, state=S)
    cuts = [0, 1, 2, 50, 51, 52, 53, 120, 150]
    parts = torch.cat([short_conv(x[i:j], w, b, state=P) for i, j in zip(cuts, cuts[1:])])
    torch.cuda.synchronize()
    assert torch.equal(whole, parts) and torch.equal(S, P) and torch.equal(S[0], x[-3:])


@types
def test_strided_and_misaligned(fmt):
    def wide(x):
        row = torch.full((x.shape[0], x.shape[1] + 5), math.nan, dtype=x.dtype, device="cuda")
        row[:, 3:3 + x.shape[1]] = x.cuda()
        return row[:, 3:3 + x.shape[1]]

    def shifted(x):
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        return y.copy_(x)
    check(fmt, 130, 64, 4, seed=14, place=wide)
    check(fmt, 70, 37, 4, seed=15, place=wide)
    check(fmt, 70, 64, 4, seed=15, place=shifted)


@types
def test_not_finite(fmt):
    """An entry that is not finite is in the outputs of its channel that have it as a factor, and in no other."""
    def spoil(x):
        x[20, 3], x[40, 5], x[60, 7] = math.nan, math.inf, float(torch.finfo(x.dtype).min) / 8
    o, want, off = check(fmt, 100, 16, 4, seed=16, change=spoil)
    hit = np.zeros((100, 16), bool)
    hit[20:24, 3] = hit[40:44, 5] = hit[60:64, 7] = True
    clean, _, _ = check(fmt, 100, 16, 4, seed=16)
    assert np.array_equal(o[~hit], clean[~hit]) and np.isnan(o[20:24, 3]).all()
    assert not np.isfinite(o[40:44, 5]).any()
    large = np.where(np.isfinite(o[60:64, 7]), o[60:64, 7], 0.0)         # (binary16 has no numbers for some)
    assert not np.isnan(o[60:64, 7]).any() and ref.within(large[large != 0], want[60:64, 7][large != 0], off[60:64, 7][large != 0], fmt) <= 0


def test_entries_past_32_bits():
    """Rows whose offsets pass 2^31 elements."""
    T, C, ld = 70, 24, 2 ** 25
    buffer = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    x, w, b = inputs(17, T, C, 4, "bf16")
    rows = buffer.as_strided((T, C), (ld, 1))
    rows.copy_(x)
    a, c = short_conv(rows, w.cuda(), b.cuda()), short_conv(x.cuda(), w.cuda(), b.cuda())
    torch.cuda.synchronize()
    assert torch.equal(a, c)


def test_offsets_out_of_range_stay_inside():
    x, w, b = (v.cuda() for v in inputs(18, 80, 16, 4, "f32"))
    a = short_conv(x, w, b, starts=i32([-50, 30, 2000]))
    c = short_conv(x, w, b, starts=i32([0, 30, 80]))
    torch.cuda.synchronize()
    assert torch.equal(a, c)


def test_stream_and_graph():
    x, w, b = (v.cuda() for v in inputs(19, 300, 72, 4, "bf16"))
    S0, starts = torch.randn(2, 3, 72, device="cuda").bfloat16(), i32([0, 170, 300])

    def once(stream=None):
        S = S0.clone()
        torch.cuda.synchronize()
        o = short_conv(x, w, b, starts=starts, state=S, stream=stream)
        torch.cuda.synchronize()
        return o, S
    want = once()
    for got in (once(), once(torch.cuda.Stream())):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    S, out = S0.clone(), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        short_conv(x, w, b, starts=starts, state=S, out=out)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        want = once()
        S.copy_(S0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(S, want[1])


def test_refusals():
    x, w, b = (v.cuda() for v in inputs(20, 12, 16, 4, "f32"))
    S, out = torch.zeros(1, 3, 16, device="cuda"), torch.empty(12, 16, device="cuda")
    good = dict(type=0, channels=16, width=4, silu=1, n_seq=1, n_states=1, n_tokens=12, d_x=x.data_ptr(), ldx=16, d_w=w.data_ptr(), d_bias=b.data_ptr(),
                d_state_in=S.data_ptr(), d_state_out=S.data_ptr(), d_out=out.data_ptr(), ldo=16)

    def call(**change):
        return lib().csb_short_conv(csb_conv_args(**{**good, **change}), None)
    assert call() == 0 and call(n_seq=0) == 0 and call(n_tokens=0) == 0 and call(d_bias=None) == 0
    for change in (dict(type=3), dict(channels=0), dict(width=0), dict(n_seq=-1), dict(n_tokens=-1), dict(n_seq=5), dict(ldx=15), dict(ldo=15),
                   dict(n_states=0), dict(d_x=None), dict(d_w=None), dict(d_out=None), dict(d_out=x.data_ptr()), dict(d_x=x.data_ptr() + 1),
                   dict(d_state_in=S.data_ptr() + 2), dict(d_w=w.data_ptr() + 2)):
        assert call(**change) == -1, change
    assert call(width=9) == -4 and call(n_tokens=1 << 31) == -4 and call(n_seq=1 << 28, n_tokens=0) == -4
    assert lib().csb_short_conv(None, None) == -1 and lib().csb_last_error().startswith(b"csb_short_conv")
    with pytest.raises(AssertionError):
        short_conv(x, w[:8], b)
    with pytest.raises(AssertionError):
        short_conv(x, w.half(), b)
    with pytest.raises(AssertionError):
        short_conv(x, w, b, state=torch.zeros(1, 4, 16, device="cuda"))
    with pytest.raises(CsbError, match="out is x"):
        short_conv(x, w, b, out=x)
    with pytest.raises(CsbError, match="leading dimension"):
        short_conv(x[:1].expand(12, 16), w, b)
    torch.cuda.synchronize()
