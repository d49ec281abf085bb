"""Calls of the operators around a recurrent layer that their documents allow and that come seldom: temperatures and logits whose differences pass binary32, states
read by several sequences, one state under two names, sequences of very different lengths, one channel and many short sequences."""
import math

import pytest
import torch

import test_gpu_sample as samples
import test_gpu_scan as scans
from paper_2005_05758_amd import block_norm, selective_scan, short_conv

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("V", [900, 30000])
def test_differences_of_logits_past_binary32(V):
    """Logits up to 3e38 of both signs, whose differences a temperature of their size makes numbers of again."""
    t = torch.Generator().manual_seed(3)
    logits = (torch.rand(6, V, generator=t) * 2 - 1) * 3e38
    r = torch.rand(6, generator=t)
    T = [1e38, 3e37, math.inf, 2e38, 3e38, 1e37]
    for numbers in (dict(), dict(top_k=[V // 2, V - 5, V // 3, 300, 40, 500]), dict(top_p=[0.9, 0.99, 0.7, 0.6, 0.97, 0.5])):
        samples.check(logits, r, temperature=T, **numbers)


def scan_inputs(seed, T, C=24, n=8):
    t = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=t)                                # noqa: E731
    return [v.cuda() for v in (rnd(T, C), 0.3 * rnd(T, C), -rnd(C, n).abs(), rnd(T, 1, n), rnd(T, 1, n))]


@pytest.mark.parametrize("T", [6, 96, 2000])
def test_one_state_for_several_sequences(T):
    """Read by all of them, kept by none: as with every one alone."""
    say(f"[edges] one state, {T} tokens")
    x, dt, A, B, C = scan_inputs(1, T)
    S = torch.randn(2, 24, 8, device="cuda")
    kept = S.clone()
    got = selective_scan(x, dt, A, B, C, state=S, state_out=None, starts=i32([0, T // 2, T]), slots=i32([1, 1]))
    halves = [selective_scan(*(v[i] if v is not A else v for v in (x, dt, A, B, C)), state=S[1:], state_out=None) for i in (slice(0, T // 2), slice(T // 2, T))]
    off = 0.0 if T == 6 else 1e-5                         # (another split into chunks)
    assert (got - torch.cat(halves)).abs().max() <= off * got.abs().max() and torch.equal(S, kept)
    w = torch.randn(24, 4, device="cuda")
    P = torch.randn(2, 3, 24, device="cuda")
    got = short_conv(x, w, state=P, state_out=None, starts=i32([0, T // 2, T]), slots=i32([1, 1]))
    halves = [short_conv(x[i], w, state=P[1:], state_out=None) for i in (slice(0, T // 2), slice(T // 2, T))]
    assert torch.equal(got, torch.cat(halves))


def test_two_sequences_that_leave_one_state():
    """They race for it: whichever it is, nothing else is touched, and the outputs do not depend on it where it is kept elsewhere."""
    say("[edges] two sequences, one state")
    x, dt, A, B, C = scan_inputs(2, 12)
    S, other = torch.zeros(3, 24, 8, device="cuda"), torch.full((3, 24, 8), 7.0, device="cuda")
    apart = torch.zeros(3, 24, 8, device="cuda")
    out = selective_scan(x, dt, A, B, C, state=S, state_out=other, starts=i32([0, 5, 12]), slots=i32([1, 1]))
    want = selective_scan(x, dt, A, B, C, state=S, state_out=apart, starts=i32([0, 5, 12]), slots=i32([0, 1]))
    assert torch.equal(out, want) and bool((other[[0, 2]] == 7.0).all())
    assert bool(((other[1] == apart[0]) | (other[1] == apart[1])).all())


def test_one_long_sequence_among_single_tokens():
    """The rule for the kernel is the mean length; a call is right whatever the lengths are."""
    lengths = [1] * 300 + [1500] + [1] * 100
    T, n = sum(lengths), 8
    say(f"[edges] lengths 1 and 1500, {T} tokens")
    x, dt, A, B, C = scan_inputs(4, T)
    at = torch.tensor([0] + lengths).cumsum(0)
    S = torch.randn(len(lengths), 24, n, device="cuda")
    alone = S[300:301].clone()
    got = selective_scan(x, dt, A, B, C, starts=at.int().cuda(), state=S)
    i = slice(300, 1800)
    want = selective_scan(x[i], dt[i], A, B[i], C[i], state=alone)
    assert (got[i] - want).abs().max() <= 1e-5 * want.abs().max() and (S[300:301] - alone).abs().max() <= 1e-5 * alone.abs().max()
    w = torch.randn(24, 4, device="cuda")
    assert torch.equal(short_conv(x, w, starts=at.int().cuda())[i], short_conv(x[i], w))


@pytest.mark.parametrize("C", [1, 8, 40])
def test_few_channels_and_many_short_sequences(C):
    say(f"[edges] 3000 sequences of {C} channels")
    t = torch.Generator().manual_seed(C)
    lengths = torch.randint(0, 60, (3000,), generator=t)
    at = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)])
    T = int(at[-1])
    x, w = torch.randn(T, C, generator=t), torch.randn(C, 4, generator=t)
    S = torch.randn(3000, 3, C, generator=t)
    state = S.cuda()
    got = short_conv(x.cuda(), w.cuda(), silu=False, starts=at.int().cuda(), state=state).cpu()
    whole = torch.zeros(T, C, dtype=torch.float64)
    new = S.clone()
    for s in range(3000):
        seq = torch.cat([S[s], x[at[s]:at[s + 1]]])
        new[s] = seq[len(seq) - 3:]
        for j in range(4):
            whole[at[s]:at[s + 1]] += w[:, j].double() * seq[j:j + int(lengths[s])].double()
    # four products and sums of numbers up to 4.5 * 4.5: 8 roundings of 2^-24 of 4 * 20
    assert (got.double() - whole).abs().max() <= 8 * 2.0 ** -24 * 4 * float(x.abs().max() * w.abs().max()) and torch.equal(state.cpu(), new)


def test_rows_of_one_token_and_one_entry():
    """Views whose strides say nothing."""
    say("[edges] one token, one entry")
    x = torch.randn(5, 64, device="cuda")
    for v in (x[2:3], x.t()[:, 2:3].t(), x[:, 7:8], x.t()[7:8].t()):
        r, n = block_norm(v, x=v, after="rms", before="rms")
        want_r, want_n = block_norm(v.contiguous(), x=v.contiguous(), after="rms", before="rms")
        assert torch.equal(r, want_r) and torch.equal(n, want_n)
    w = torch.randn(64, 4, device="cuda")
    assert torch.equal(short_conv(x[2:3], w), short_conv(x[2:3].clone(), w))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_that_go_past_the_caches(dtype):
    """A norm between products of more than 32 MiB: what it leaves is what its halves, which are below that, leave."""
    say("[edges] 4100 tokens of 4104 entries")
    T, W = 4100, 4104
    y, x = torch.randn(W, T, device="cuda"), torch.randn(T, W, device="cuda").to(dtype)
    whole, halves = [], []
    for into, parts in ((whole, [slice(0, T)]), (halves, [slice(0, T // 2), slice(T // 2, T)])):
        r, n = torch.empty_like(x), torch.empty(W, T, device="cuda", dtype=dtype)
        for p in parts:
            block_norm(y[:, p].t(), x=x[p], before="rms", out=r[p], normed=n[:, p].t())
        into += [r, n]
    # sums of another order are 2^-50 off: results are the same number, or one of two neighbours where they lie between them
    assert torch.equal(whole[0], halves[0])
    off = (whole[1].float() - halves[1].float()).abs()
    assert (off <= torch.finfo(dtype).eps * halves[1].float().abs()).all() and int((off > 0).sum()) <= T * W // 10000


def odd_views(dev):
    """Rows of tokens at odd strides, from the second element of a buffer on."""
    out = []
    for v in dev:
        if v is None or v.dim() < 2 or v is dev[2]:     # (A is whole)
            out.append(v)
            continue
        width = v[0].numel()
        buf = torch.zeros(v.shape[0] * (width + 7) + 8, dtype=v.dtype, device="cuda")
        rows = buf[1:1 + v.shape[0] * (width + 7)].view(v.shape[0], width + 7)[:, :width]
        rows.copy_(v.reshape(v.shape[0], width))
        out.append(rows if v.dim() == 2 else rows.unflatten(1, tuple(v.shape[1:])))
    return out


@pytest.mark.parametrize("fmt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("place", [None, odd_views])
def test_scans_of_whole_tiles_of_channels(fmt, place):
    """64 channels of a group and all of their numbers: chunks of one tile, of several, whole sequences of several tiles, and what is left of them."""
    scans.check(fmt, 700, 192, 1, 16, seed=41, place=place)
    scans.check(fmt, 4200, 64, 1, 16, lengths=[4197], seed=42, place=place)
    scans.check(fmt, 300, 128, 2, 64, lengths=[150, 33, 64, 1, 20, 32], seed=43, place=place, softplus=False, without=(6,))
    lengths = [40, 64, 97, 33, 32, 31, 0, 128, 70] * 3
    scans.check(fmt, sum(lengths), 64 * 40, 1, 16, lengths=lengths, lens=[n - (n > 50) for n in lengths], seed=44, place=place)


@pytest.mark.parametrize("fmt,V", [("f32", 24576), ("f32", 24577), ("bf16", 49152), ("bf16", 49153), ("f16", 4096), ("f32", 8193), ("bf16", 16385)])
def test_rows_of_which_much_is_kept(fmt, V):
    """Flat and even rows, whose kept tokens fit into no list, at the sizes where the forms change."""
    t = torch.Generator().manual_seed(V)
    r = torch.tensor([0.0, 0.3, 0.999, 0.5, 0.7, 1 - 2.0 ** -24])
    flat = (0.5 * torch.randn(6, V, generator=t)).to(samples.TYPES[fmt])
    flat[4] = 1.25                                       # all equal
    flat[5, ::2] = -math.inf
    samples.check(flat, r)
    samples.check(flat, r, top_p=[0.9, 0.999, 0.5, 0.01, 0.6, 0.97])
    samples.check(flat, r, top_k=[V - 1, 5000, 4096, 4097, 2000, V // 2 - 3])
    samples.check(flat, r, top_k=[V // 2, 3000, 300, 257, 256, 0], top_p=[0.99, 0.9, 0.8, 0.5, 0.3, 1.5], min_p=[0.01, 0.1, 0.3, 0.0, 0.5, 0.2], temperature=[0.3, 0.5, 1.0, 2.0, 1.0, 0.7])
    samples.check(flat, r, min_p=[0.01, 0.1, 0.3, 0.9, 1.0, 0.2])
