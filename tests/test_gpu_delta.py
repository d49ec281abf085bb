"""The gated delta rule (csb_delta_recurrent, csb_delta_chunked) against its definition in 64 bits on the host.

Tolerances.  A token's step forms sums of dk products in binary32 and u, S and o from them; with keys of length one and
beta in [0, 2] no later step makes an error larger (|1 - beta k k^T| <= 1), so errors add up over the tokens like
independent ones.  STATE = 16 sqrt(256) 2^-24 of the largest state entry covers the widest dk here and the few hundred
tokens of a case; `out` adds half a unit in the last place of its type."""
import math
import sys

import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_2005_05758_amd import delta_chunked, delta_recurrent
from paper_2005_05758_amd.binding import CsbError, csb_delta_args, lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
STATE = 16 * math.sqrt(256) * 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit in the last place, of the value
FORMS = {"recurrent": delta_recurrent, "chunked": delta_chunked}
both = pytest.mark.parametrize("form", sorted(FORMS))


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def inputs(seed, T, HK, HV, DK, DV, fmt, alike=0.0, strong=1.0):
    """Keys and queries of length one (`alike`: how much they share), decays of a few per mille to e^-strong."""
    t = torch.Generator().manual_seed(seed)
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, generator=t) * (1 - alike) + alike, dim=-1)   # noqa: E731
    q, k, v = unit(T, HK, DK), unit(T, HK, DK), torch.randn(T, HV, DV, generator=t)
    g = -strong * torch.rand(T, HV, generator=t) ** 3
    beta = 2.0 * torch.rand(T, HV, generator=t) if alike else torch.sigmoid(torch.randn(T, HV, generator=t))
    return [x.to(TYPES[fmt]) for x in (q, k, v)] + [g, beta]


def check(form, fmt, T, HK, HV, DK, DV, lengths=None, lens=None, slots=None, n_states=None, seed=0, state=True, keep=True, place=None,
          change=None, **kw):
    say(f"[delta] {form} {fmt} T={T} heads {HK}/{HV} {DK}x{DV} lengths={lengths} lens={lens} slots={slots} {place or ''} {kw}")
    q, k, v, g, beta = inputs(seed, T, HK, HV, DK, DV, fmt, **kw)
    if change:
        change(q, k, v, g, beta)
    N = len(lengths) if lengths is not None else 1
    first = np.concatenate([[0], np.cumsum(lengths)]).astype(int) if lengths is not None else np.array([0, T])
    ranges = [(first[i], first[i] + min(max(lens[i], 0), first[i + 1] - first[i]) if lens is not None else first[i + 1]) for i in range(N)]
    n_states = n_states or N
    S0 = torch.randn(n_states, HV, DK, DV, generator=torch.Generator().manual_seed(seed + 1)) if state else None
    where = [s if 0 <= s < n_states else -1 for s in slots] if slots is not None else list(range(N))
    scale = DK ** -0.5
    ro, rs = ref.delta(*(ref.widen(x) for x in (q, k, v, g, beta)), scale, ranges, where if state else [-1] * N,
                       ref.widen(S0) if state else np.zeros((n_states, HV, DK, DV)))
    dev = [x.cuda() for x in (q, k, v, g, beta)]
    if place:
        dev = place(dev)
    out = torch.full((T, HV, DV), 7.0, dtype=TYPES[fmt], device="cuda")
    Sd = S0.cuda() if state else None
    before = Sd.clone() if state else None
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda") if x is not None else None     # noqa: E731
    got = FORMS[form](*dev, scale=scale, starts=i32(list(first)) if lengths is not None else None, lens=i32(lens), slots=i32(slots),
                      state=Sd, out=out, **({} if keep else {"state_out": None}))
    torch.cuda.synchronize()
    assert got is out
    o = out.cpu().double().numpy()
    there = ~np.isnan(ro)
    if change is None:
        assert np.array_equal(o[~there], np.full((~there).sum(), 7.0)), "tokens that no sequence takes are not written"
        if there.any():
            far = np.abs(o - ro)[there] - (HALF[fmt] * np.abs(ro[there]) + STATE * np.abs(ro[there]).max() + 2.0 ** -25)
            assert far.max() <= 0, (far.max(), np.abs(ro[there]).max())
        if state:
            s = Sd.cpu().double().numpy()
            if keep:
                assert np.abs(s - rs).max() <= STATE * max(1.0, np.abs(rs).max()), np.abs(s - rs).max()
                for i in set(range(n_states)) - set(where):
                    assert torch.equal(Sd[i], before[i])
            else:
                assert torch.equal(Sd, before)
    return o, ro, Sd, rs


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("T,HK,HV,DK,DV", [(1, 1, 1, 1, 1), (2, 1, 3, 16, 16), (64, 2, 2, 64, 64), (65, 1, 2, 128, 128), (63, 1, 1, 33, 5), (130, 2, 4, 100, 48),
                                           (129, 1, 1, 200, 70), (70, 1, 2, 256, 130), (200, 1, 1, 96, 80)])
def test_one_sequence(form, fmt, T, HK, HV, DK, DV):
    check(form, fmt, T, HK, HV, DK, DV, seed=T + DK)


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_packed_sequences(form, fmt):
    lengths = [1, 0, 64, 3, 128, 65, 0, 0, 31, 2]
    check(form, fmt, sum(lengths), 2, 4, 48, 32, lengths=lengths, seed=3)
    # states anywhere in a pool, some requests without one; fewer tokens taken than there are
    check(form, fmt, sum(lengths) + 5, 1, 2, 64, 20, lengths=lengths, slots=[11, 3, -1, 0, 99, 7, 5, 2, 1, -2], n_states=12, seed=4)
    check(form, fmt, sum(lengths), 1, 2, 64, 20, lengths=lengths, lens=[1, 0, 63, -4, 65, 99, 2, 0, 0, 1], seed=5)


@both
def test_many_sequences(form):
    g = np.random.default_rng(1)
    lengths = [int(x) for x in g.integers(0, 4, 700)]
    check(form, "bf16", sum(lengths), 1, 1, 16, 16, lengths=lengths, slots=[int(x) for x in g.permutation(700)], seed=6)


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_many_wide_sequences(form, fmt):
    """Enough sequences and heads for every CU, rows of 65 to 128 elements, the last columns alone in their workgroup."""
    g = np.random.default_rng(2)
    lengths = [int(x) for x in g.integers(0, 91, 130)]
    check(form, fmt, sum(lengths), 1, 2, 100, 48, lengths=lengths, slots=[int(x) for x in g.permutation(133)[:130]], n_states=133, seed=20)


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("DK", [3, 7, 8, 9, 15, 31, 65, 121, 128])
def test_widths(form, fmt, DK):
    """Rows that end anywhere in a word; enough sequences and heads for every CU."""
    g = np.random.default_rng(DK)
    lengths = [int(x) for x in g.integers(0, 70, 66)]
    check(form, fmt, sum(lengths), 2, 4, DK, 20, lengths=lengths, seed=DK)


@both
def test_states_from_zero_and_not_kept(form):
    check(form, "bf16", 90, 1, 2, 64, 32, lengths=[70, 20], seed=7, state=False)
    check(form, "f16", 90, 1, 2, 64, 32, lengths=[70, 20], seed=8, keep=False)


@both
def test_state_into_another_buffer(form):
    """The last states go to a second buffer; a sequence of no tokens takes its state over as it is."""
    q, k, v, g, beta = (x.cuda() for x in inputs(9, 80, 1, 2, 32, 24, "f32"))
    S = torch.randn(3, 2, 32, 24, device="cuda")
    into, starts = torch.full_like(S, 5.0), torch.tensor([0, 70, 70, 80], dtype=torch.int32, device="cuda")
    a = FORMS[form](q, k, v, g, beta, starts=starts, state=S, state_out=into)
    keep = S.clone()
    b = FORMS[form](q, k, v, g, beta, starts=starts, state=S)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(into, S) and torch.equal(into[1], keep[1]) and not torch.equal(into[0], keep[0])


@both
@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_keys_alike(form, fmt):
    """Keys that are nearly the same and steps of up to 2: the corrections within a chunk are as large as they get."""
    check(form, fmt, 150, 1, 2, 64, 16, seed=10, alike=0.9, strong=0.01)


@both
def test_decays(form):
    """Decays that forget at once, that lose everything over a few tokens, and none at all; steps of 0."""
    def forget(q, k, v, g, beta):
        g[5] = -math.inf
        g[66:69] = -math.inf
        g[100:110] = -90.0
        g[20:40] = 0.0
        beta[30:33] = 0.0
    o, ro, S, rs = check(form, "f32", 140, 1, 1, 32, 16, seed=11, change=forget)
    assert np.abs(o - ro).max() <= STATE * np.abs(ro).max() + 2.0 ** -25
    assert np.abs(S.cpu().double().numpy() - rs).max() <= STATE * max(1.0, np.abs(rs).max())

    def long_forgotten(q, k, v, g, beta):                # large decays before tokens that hardly decay: differences of their sums count
        g[:40] = -60.0
        g[40:] = -1e-3
    o, ro, S, rs = check(form, "f32", 140, 1, 1, 32, 16, seed=12, change=long_forgotten)
    assert np.abs(o - ro).max() <= STATE * np.abs(ro).max() + 2.0 ** -25


@both
def test_not_finite(form):
    """A token with an infinite or NaN entry spoils its own sequence and head from there on, and nothing else."""
    def spoil(q, k, v, g, beta):
        v[70, 1, 3] = math.inf
        k[101, 0, 2] = math.nan
    lengths = [64, 36, 40]
    o, ro, S, rs = check(form, "bf16", 140, 2, 4, 32, 16, lengths=lengths, seed=13, change=spoil)
    clean, _, Sc, _ = check(form, "bf16", 140, 2, 4, 32, 16, lengths=lengths, seed=13)
    hit = np.zeros((140, 4), bool)
    hit[64:100, 1] = True                                # sequence 1, value head 1 (earlier tokens of a chunk may go too)
    hit[100:140, 0:2] = True                             # sequence 2, the value heads of key head 0
    assert np.array_equal(o[~hit], clean[~hit]) and np.isfinite(o[~hit]).all()
    assert np.isfinite(o[64:70]).all()                   # tokens before it
    assert not np.isfinite(o[70:100, 1, 3]).any() and not np.isfinite(o[101:, 0:2]).any()
    S, Sc = S.cpu(), Sc.cpu()
    assert torch.equal(S[0], Sc[0]) and torch.equal(S[1, [0, 2, 3]], Sc[1, [0, 2, 3]]) and torch.equal(S[2, 2:], Sc[2, 2:])


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_not_finite_gates_and_queries(form, fmt):
    """A gate or a step that is NaN spoils its value head from its token on, a query its token's output only."""
    def spoil(q, k, v, g, beta):
        g[80, 0] = math.nan
        beta[130, 1] = math.nan
        beta[150, 1] = math.inf
        q[20, 0, 7] = math.nan
    lengths = [100, 70]
    o, _, S, _ = check(form, fmt, 170, 1, 2, 72, 40, lengths=lengths, seed=21, change=spoil)
    clean, _, Sc, _ = check(form, fmt, 170, 1, 2, 72, 40, lengths=lengths, seed=21)
    hit = np.zeros((170, 2), bool)
    hit[80:100, 0] = hit[130:, 1] = hit[20] = True
    assert not np.isfinite(o[hit]).any()
    near = np.zeros((170, 2), bool)                      # tokens of the same chunk before it: right, their bits may differ
    near[64:80, 0] = near[100:130, 1] = True
    assert np.array_equal(o[~hit & ~near], clean[~hit & ~near]) and np.isfinite(o[near]).all()
    S, Sc = S.cpu(), Sc.cpu()
    assert torch.equal(S[0, 1], Sc[0, 1]) and torch.equal(S[1, 0], Sc[1, 0])
    assert not torch.isfinite(S[0, 0]).any() and not torch.isfinite(S[1, 1]).any()


@both
@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_strided_and_misaligned(form, fmt):
    def fused(dev):                                      # q, k and v as parts of one projection's rows
        q, k, v, g, beta = dev
        T = q.shape[0]
        row = torch.full((T, q[0].numel() * 2 + v[0].numel() + 3), math.nan, dtype=q.dtype, device="cuda")
        at, parts = 0, []
        for x in (q, k, v):
            part = row[:, at:at + x[0].numel()].view(T, *x.shape[1:]) if False else row[:, at:at + x[0].numel()].unflatten(1, x.shape[1:])
            part.copy_(x)
            parts.append(part)
            at += x[0].numel()
        gb = torch.full((T, 2 * g.shape[1] + 1), math.nan, device="cuda")
        gb[:, :g.shape[1]] = g
        gb[:, g.shape[1]:-1] = beta
        return parts + [gb[:, :g.shape[1]], gb[:, g.shape[1]:-1]]

    def shifted(dev):                                    # bases aligned to one element only
        moved = []
        for x in dev:
            y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
            y.copy_(x)
            moved.append(y)
        return moved
    check(form, fmt, 130, 2, 2, 64, 64, seed=14, place=fused)
    check(form, fmt, 70, 1, 2, 32, 48, seed=15, place=shifted)


@both
def test_other_stream_and_repeats(form):
    """The same bits on every call, on another stream, and replayed from a graph with new contents."""
    q, k, v, g, beta = (x.cuda() for x in inputs(16, 300, 2, 4, 64, 64, "bf16"))
    S0 = torch.randn(2, 4, 64, 64, device="cuda")
    starts = torch.tensor([0, 170, 300], dtype=torch.int32, device="cuda")
    call = FORMS[form]

    def once(stream=None):
        S = S0.clone()
        torch.cuda.synchronize()
        o = call(q, k, v, g, beta, starts=starts, state=S, stream=stream)
        torch.cuda.synchronize()
        return o, S
    want = once()
    side = torch.cuda.Stream()
    for got in (once(), once(side)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    S, out = S0.clone(), torch.empty_like(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(q, k, v, g, beta, starts=starts, state=S, out=out)
    for i in range(3):
        v.copy_(torch.randn_like(v))
        want = once()
        S.copy_(S0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(S, want[1])


@both
def test_states_past_32_bits(form):
    """A pool of states of more than 2^31 elements: the last one is found."""
    n = 2 ** 31 // (16 * 128 * 128) + 2
    S = torch.empty(n, 16, 128, 128, device="cuda")
    S[-1] = 0.1
    S[0] = 0.2
    q, k, v, g, beta = (x.cuda() for x in inputs(17, 70, 4, 16, 128, 128, "bf16"))
    small = S[-1:].clone()
    o = FORMS[form](q, k, v, g, beta, state=S, slots=torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
    o2 = FORMS[form](q, k, v, g, beta, state=small)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(S[-1], small[0]) and bool((S[0] == 0.2).all())


@both
def test_offsets_out_of_range_stay_inside(form):
    """Offsets are device memory: what lies outside [0, tokens] is taken as the nearer end."""
    q, k, v, g, beta = (x.cuda() for x in inputs(18, 80, 1, 2, 32, 16, "f32"))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
    a = FORMS[form](q, k, v, g, beta, starts=i32([-50, 30, 2000]))
    b = FORMS[form](q, k, v, g, beta, starts=i32([0, 30, 80]))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_refusals():
    q, k, v, g, beta = (x.cuda() for x in inputs(19, 12, 2, 4, 32, 16, "f32"))
    S, out = torch.zeros(1, 4, 32, 16, device="cuda"), torch.empty(12, 4, 16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    good = dict(type=0, heads_k=2, heads_v=4, dk=32, dv=16, n_seq=1, n_tokens=12, d_q=q.data_ptr(), d_k=k.data_ptr(), d_v=v.data_ptr(),
                ldq=64, ldk=64, ldv=64, d_g=g.data_ptr(), d_beta=beta.data_ptr(), ldg=4, ldbeta=4, d_state_in=S.data_ptr(),
                d_state_out=S.data_ptr(), n_states=1, scale=1.0, d_out=out.data_ptr(), ldo=64)

    def calls(**change):
        a = csb_delta_args(**{**good, **change})
        return (lib().csb_delta_recurrent(a, None), lib().csb_delta_chunked(a, ws.data_ptr(), None))
    assert calls() == (0, 0) and calls(n_seq=0) == (0, 0) and calls(n_tokens=0) == (0, 0)
    assert lib().csb_delta_workspace_bytes(csb_delta_args(**good)) <= ws.numel()
    for change in (dict(type=3), dict(heads_k=0), dict(heads_k=3), dict(heads_v=0), dict(dk=0), dict(dv=0), dict(n_seq=-1), dict(n_tokens=-1),
                   dict(n_seq=5), dict(ldq=63), dict(ldk=63), dict(ldv=63), dict(ldo=63), dict(ldg=3), dict(ldbeta=3), dict(n_states=0),
                   dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_g=None), dict(d_beta=None), dict(d_out=None),
                   dict(d_q=q.data_ptr() + 1), dict(d_state_in=S.data_ptr() + 2)):
        assert calls(**change) == (-1, -1), change
    assert calls(dk=257, ldq=1024, ldk=1024) == (-4, -4)
    assert calls(n_seq=1 << 30, n_tokens=0)[0] == -4
    assert lib().csb_delta_recurrent(None, None) == -1 and lib().csb_delta_chunked(None, None, None) == -1
    assert lib().csb_last_error().startswith(b"csb_delta_chunked")
    with pytest.raises(AssertionError):
        delta_chunked(q, k[:, :1], v, g, beta)
    with pytest.raises(AssertionError):
        delta_recurrent(q.half(), k, v, g, beta)
    with pytest.raises(CsbError):
        delta_recurrent(q, k, v, g, beta, slots=torch.zeros(5, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


def test_refusals_of_the_chunked_form():
    """Strides and widths whose offsets would pass 32 bits, more workgroups than a launch takes."""
    q, k, v, g, beta = (x.cuda() for x in inputs(22, 12, 2, 4, 32, 16, "bf16"))
    out, ws = torch.empty(12, 4, 16, device="cuda", dtype=torch.bfloat16), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    good = dict(type=2, heads_k=2, heads_v=4, dk=32, dv=16, n_seq=1, n_tokens=12, d_q=q.data_ptr(), d_k=k.data_ptr(), d_v=v.data_ptr(),
                ldq=64, ldk=64, ldv=64, d_g=g.data_ptr(), d_beta=beta.data_ptr(), ldg=4, ldbeta=4, scale=1.0, d_out=out.data_ptr(), ldo=64)

    def call(d_ws=ws.data_ptr(), **change):
        return lib().csb_delta_chunked(csb_delta_args(**{**good, **change}), d_ws, None)
    assert call() == 0
    for name in ("ldq", "ldk", "ldv", "ldo"):
        assert call(**{name: 1 << 23}) == -4, name
    assert call(dv=(1 << 20) + 1, ldv=1 << 22 | 64, ldo=1 << 22 | 64) == -4
    assert call(n_seq=1 << 24, n_tokens=0) == -4
    assert call(d_ws=None) == -1 and call(d_ws=ws.data_ptr() + 16) == -1
    torch.cuda.synchronize()
