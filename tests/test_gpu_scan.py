"""The selective state space scan (csb_selective_scan) against its definition in 64 bits on the host, with bounds that follow the
recurrence (layer_reference.scan)."""
import math
import sys

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2005_05758_amd import selective_scan
from paper_2005_05758_amd.binding import CsbError, csb_scan_args, lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
types = pytest.mark.parametrize("fmt", sorted(TYPES))


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if x is not None else None


def inputs(seed, T, C, G, n, fmt):
    """x, dt, A, B, C, D, z, dt_bias: steps of 0.001 to 0.1, decays from hardly any to half a token's."""
    t = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    typ = TYPES[fmt]
    step = torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(C, generator=t))
    return [rnd(T, C).to(typ), (0.5 * rnd(T, C)).to(typ), -8.0 * torch.rand(C, n, generator=t), rnd(T, G, n).to(typ), rnd(T, G, n).to(typ), rnd(C),
            rnd(T, C).to(typ), torch.log(torch.expm1(step))]


def call(ins, **kw):
    x, dt, A, B, C, D, z, bias = (v.cuda() if v is not None else None for v in ins)
    return selective_scan(x, dt, A, B, C, D=D, z=z, dt_bias=bias, **kw)


def check(fmt, T, C, G, n, lengths=None, lens=None, slots=None, n_states=None, seed=0, softplus=True, without=(), state=True, keep=True, place=None,
          change=None):
    say(f"[scan] {fmt} T={T} C={C}/{G} n={n} lengths={lengths} lens={lens} slots={slots} {place or ''} without={without}")
    ins = inputs(seed, T, C, G, n, fmt)
    if change:
        change(*ins)
    if not softplus:
        ins[1] = (0.05 * ins[1].float().abs()).to(TYPES[fmt])
        ins[7] = 0.01 * ins[7].abs()
    for i in without:
        ins[i] = None
    N = len(lengths) if lengths is not None else 1
    first = np.concatenate([[0], np.cumsum(lengths)]).astype(int) if lengths is not None else np.array([0, T])
    ranges = [(first[i], first[i] + min(max(lens[i], 0), first[i + 1] - first[i]) if lens is not None else first[i + 1]) for i in range(N)]
    n_states = n_states or N
    S0 = torch.randn(n_states, C, n, generator=torch.Generator().manual_seed(seed + 1))
    where = [s if 0 <= s < n_states else -1 for s in slots] if slots is not None else list(range(N))
    wide = [ref.widen(v) if v is not None else None for v in ins]
    with np.errstate(all="ignore"):
        want, off, ws, ws_off = ref.scan(*wide[:5], wide[5] if wide[5] is not None else np.zeros(C), wide[6], wide[7] if wide[7] is not None else np.zeros(C),
                                         softplus, ranges, where if state else [-1] * N, ref.widen(S0), fmt)
    dev = [v.cuda() if v is not None else None for v in ins]
    if place:
        dev = place(dev)
    S = S0.cuda() if state else None
    out = torch.full((T, C), 7.0, dtype=TYPES[fmt], device="cuda")
    got = selective_scan(*dev[:5], D=dev[5], z=dev[6], dt_bias=dev[7], softplus=softplus, starts=i32([int(f) for f in first]) if lengths is not None else None,
                         lens=i32(lens), slots=i32(slots), state=S, out=out, **({} if keep else {"state_out": None}))
    torch.cuda.synchronize()
    assert got is out
    o = ref.widen(out)
    if change is None:
        there = ~np.isnan(want)
        assert (o[~there] == 7.0).all(), "tokens that no sequence takes are not written"
        assert ref.within(o, want, off, fmt) <= 0
        if state and keep:
            assert ref.within(ref.widen(S), ws, ws_off, "f32") <= 0
            for i in set(range(n_states)) - set(where):
                assert torch.equal(S[i].cpu(), S0[i])
        elif state:
            assert torch.equal(S.cpu(), S0)
    return o, want, off, S, ws


@types
@pytest.mark.parametrize("T,C,G,n", [(1, 1, 1, 1), (1, 64, 1, 16), (2, 3, 1, 5), (4, 70, 1, 16), (33, 66, 2, 17), (64, 130, 1, 32), (65, 24, 3, 9), (100, 200, 4, 64),
                                     (31, 65, 1, 65), (70, 16, 2, 128), (32, 5, 5, 3)])
def test_one_sequence(fmt, T, C, G, n):
    check(fmt, T, C, G, n, seed=T + C)


@types
@pytest.mark.parametrize("n", [1, 7, 8, 9, 16, 17, 32, 33, 60, 64, 65, 128])
def test_few_tokens(fmt, n):
    """Decoding: a few tokens of every request, of drafts of different lengths."""
    check(fmt, 11, 70, 2, n, lengths=[1, 4, 0, 2, 3, 1], slots=[5, 0, 3, -1, 7, 1], n_states=8, seed=n)
    check(fmt, 12, 130, 1, n, lengths=[4, 4, 4], lens=[1, 4, 0], seed=n + 1)


@types
def test_packed_sequences(fmt):
    lengths = [1, 0, 64, 3, 128, 65, 0, 0, 31, 2]
    check(fmt, sum(lengths), 70, 2, 16, lengths=lengths, seed=3)
    check(fmt, sum(lengths) + 5, 33, 1, 10, lengths=lengths, slots=[11, 3, -1, 0, 99, 7, 5, 2, 1, -2], n_states=12, seed=4)
    check(fmt, sum(lengths), 20, 1, 20, lengths=lengths, lens=[1, 0, 63, -4, 65, 99, 2, 0, 0, 1], seed=5)


@types
@pytest.mark.parametrize("n", [16, 7, 40])
def test_long_sequences(fmt, n):
    """Long enough for chunks (256 tokens a sequence on average), among them sequences of none, of one and of many; ends at a chunk's end and one beyond."""
    check(fmt, 1500, 70, 2, n, seed=30)
    lengths = [1, 0, 1024, 129, 128, 2000, 0, 127, 400]
    check(fmt, sum(lengths), 24, 1, n, lengths=lengths, slots=[8, 7, 6, -1, 4, 3, 2, 1, 0], seed=31)
    check(fmt, sum(lengths), 24, 1, n, lengths=lengths, lens=[9, 9, 1000, 1, 0, 256, 0, 127, 257], seed=32)


def test_many_sequences():
    g = np.random.default_rng(1)
    lengths = [int(v) for v in g.integers(0, 4, 700)]
    check("bf16", sum(lengths), 16, 1, 8, lengths=lengths, slots=[int(v) for v in g.permutation(700)], seed=6)


@pytest.mark.parametrize("T", [90, 700])
def test_forms(T):
    lengths = [T - 20, 20]
    check("f32", T, 33, 1, 16, lengths=lengths, seed=7, state=False)
    check("f16", T, 33, 1, 16, lengths=lengths, seed=8, keep=False)
    check("bf16", T, 33, 1, 16, lengths=lengths, seed=8, softplus=False)
    for without in ((5,), (6,), (7,), (5, 6, 7)):
        check("bf16", T, 33, 1, 12, lengths=lengths, seed=9, without=without)


@pytest.mark.parametrize("T", [80, 900])
@types
def test_state_into_another_buffer(fmt, T):
    ins = inputs(9, T, 40, 1, 16, fmt)
    S = torch.randn(3, 40, 16, device="cuda")
    into, starts, keep = torch.full_like(S, 5.0), i32([0, T - 10, T - 10, T]), S.clone()
    a = call(ins, starts=starts, state=S, state_out=into)
    assert torch.equal(S, keep)
    b = call(ins, starts=starts, state=S)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(into, S) and torch.equal(into[1], keep[1]) and not torch.equal(into[0], keep[0])


@pytest.mark.parametrize("T", [70, 1000])
def test_out_in_place(T):
    """Outputs over x, the steps or the gate."""
    for i in (0, 1, 6):
        ins = [v.cuda() for v in inputs(11, T, 70, 1, 16, "bf16")]
        want = call(ins)
        got = call(ins, out=ins[i])
        torch.cuda.synchronize()
        assert got is ins[i] and torch.equal(got, want)


@types
def test_strided_and_misaligned(fmt):
    def fused(dev):                                      # parts of one projection's rows
        x, dt, A, B, C, D, z, bias = dev
        T, ch = x.shape
        G, n = B.shape[1:]
        row = torch.full((T, 3 * ch + 2 * G * n + 3), math.nan, dtype=x.dtype, device="cuda")
        at, parts = 1, []
        for v in (x, z, dt, B, C):
            w = v[0].numel()
            part = row[:, at:at + w]
            part.copy_(v.flatten(1))
            parts.append(part if v.dim() == 2 else part.unflatten(1, (G, n)))
            at += w
        return [parts[0], parts[2], A, parts[3], parts[4], D, parts[1], bias]

    def shifted(dev):                                    # bases aligned to one element only
        return [torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")[1:].view(v.shape).copy_(v) for v in dev]
    check(fmt, 70, 64, 2, 16, seed=14, place=fused)
    check(fmt, 600, 37, 1, 16, seed=15, place=fused)
    check(fmt, 70, 64, 1, 16, seed=15, place=shifted)
    check(fmt, 70, 37, 1, 10, seed=15, place=shifted)


@pytest.mark.parametrize("T", [140, 900])
@pytest.mark.parametrize("n", [16, 10])
def test_not_finite(T, n):
    """What is not finite spoils its channel (B and C: their group's; C: its token only), from its token on."""
    lengths = [T - 40, 40]

    def spoil(x, dt, A, B, C, D, z, bias):
        x[70, 3], dt[90, 5], z[30, 7] = math.inf, math.nan, math.nan
        C[20, 0, 2] = math.nan
        B[T - 20, 1, 1] = math.inf
    o, want, _, S, _ = check("bf16", T, 12, 2, n, lengths=lengths, seed=13, change=spoil)
    clean, _, _, Sc, _ = check("bf16", T, 12, 2, n, lengths=lengths, seed=13)
    hit = np.zeros((T, 12), bool)
    hit[70:T - 40, 3] = hit[90:T - 40, 5] = hit[30, 7] = hit[20, 0:6] = hit[T - 20:, 6:12] = True
    assert np.array_equal(o[~hit], clean[~hit]) and np.isfinite(o[~hit]).all()
    assert not np.isfinite(o[70, 3]) and np.isnan(o[90:T - 40, 5]).all() and np.isnan(o[30, 7]) and np.isnan(o[20, 0:6]).all()
    S, Sc = S.cpu(), Sc.cpu()
    rest = [c for c in range(12) if c not in (3, 5)]
    assert torch.equal(S[0, rest], Sc[0, rest]) and torch.equal(S[1, :6], Sc[1, :6]) and not torch.isfinite(S[1, 6:, 1]).any()


@types
@pytest.mark.parametrize("T", [100, 800])
def test_steps_at_their_ends(fmt, T):
    """Steps that forget everything at once and steps of nothing."""
    def extreme(x, dt, A, B, C, D, z, bias):
        dt[20:25], dt[40:60], dt[61] = 300.0, -60.0, -math.inf
        A[:, 0] = 0.0
    o, want, off, S, ws = check(fmt, T, 20, 1, 16, seed=16, change=extreme)
    assert np.isfinite(want).all() and np.isfinite(o).all()
    assert ref.within(o, want, np.where(np.isnan(off), np.abs(want), off), fmt) <= 0


def test_large_finite_numbers():
    """Inputs of the lowest value are numbers like others where their products with the step are."""
    def lowest(x, dt, A, B, C, D, z, bias):
        x[10, 2] = float(torch.finfo(torch.float32).min)
        B[10] = 0.5
        D[2] = 0.5
    o, want, off, _, _ = check("f32", 60, 8, 1, 16, seed=17, change=lowest)
    assert np.isfinite(want).all() and np.isfinite(o).all() and ref.within(o, want, off, "f32") <= 0


@pytest.mark.parametrize("T", [300, 2000])
def test_other_stream_and_repeats(T):
    """The same bits on every call, on another stream, and replayed from a graph with new contents."""
    ins = [v.cuda() for v in inputs(18, T, 200, 2, 16, "bf16")]
    S0, starts = torch.randn(2, 200, 16, device="cuda"), i32([0, T // 3, T])

    def once(stream=None):
        S = S0.clone()
        torch.cuda.synchronize()
        o = call(ins, starts=starts, state=S, stream=stream)
        torch.cuda.synchronize()
        return o, S
    want = once()
    for got in (once(), once(torch.cuda.Stream())):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    S, out = S0.clone(), torch.empty_like(ins[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(ins, starts=starts, state=S, out=out)
    for _ in range(3):
        ins[0].copy_(torch.randn_like(ins[0]))
        want = once()
        S.copy_(S0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(S, want[1])


def test_states_past_32_bits():
    """A pool of states of more than 2^31 numbers: the last one is found."""
    n = 2 ** 31 // (4096 * 16) + 2
    S = torch.empty(n, 4096, 16, device="cuda")
    S[-1], S[0] = 0.1, 0.2
    ins = inputs(19, 5, 4096, 1, 16, "bf16")
    small = S[-1:].clone()
    a, b = call(ins, state=S, slots=i32([n - 1])), call(ins, state=small)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(S[-1], small[0]) and bool((S[0] == 0.2).all())


@pytest.mark.parametrize("T", [80, 900])
def test_offsets_out_of_range_stay_inside(T):
    ins = inputs(20, T, 24, 1, 16, "f32")
    a, b = call(ins, starts=i32([-50, 30, 20000])), call(ins, starts=i32([0, 30, T]))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_refusals():
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in inputs(21, 12, 16, 2, 8, "f32"))
    S, out = torch.zeros(1, 16, 8, device="cuda"), torch.empty(12, 16, device="cuda")
    good = dict(type=0, channels=16, groups=2, n=8, softplus=1, n_seq=1, n_tokens=12, d_x=x.data_ptr(), d_dt=dt.data_ptr(), d_z=z.data_ptr(), d_B=B.data_ptr(),
                d_C=C.data_ptr(), ldx=16, lddt=16, ldz=16, ldB=16, ldC=16, d_A=A.data_ptr(), d_D=D.data_ptr(), d_dt_bias=bias.data_ptr(),
                d_state_in=S.data_ptr(), d_state_out=S.data_ptr(), n_states=1, d_out=out.data_ptr(), ldo=16)

    def rc(d_ws=None, **change):
        return lib().csb_selective_scan(csb_scan_args(**{**good, **change}), d_ws, None)
    assert rc() == 0 and rc(n_seq=0) == 0 and rc(n_tokens=0) == 0 and rc(d_z=None, ldz=0) == 0 and rc(d_D=None, d_dt_bias=None) == 0
    for change in (dict(type=3), dict(channels=0), dict(groups=0), dict(groups=3), dict(n=0), dict(n_seq=-1), dict(n_tokens=-1), dict(n_seq=5), dict(ldx=15),
                   dict(lddt=15), dict(ldz=15), dict(ldB=15), dict(ldC=15), dict(ldo=15), dict(n_states=0), dict(d_x=None), dict(d_dt=None), dict(d_A=None),
                   dict(d_B=None), dict(d_C=None), dict(d_out=None), dict(d_x=x.data_ptr() + 1), dict(d_state_in=S.data_ptr() + 2)):
        assert rc(**change) == -1, change
    assert rc(n=129, ldB=1024, ldC=1024) == -4 and rc(n_tokens=1 << 31) == -4 and rc(n_seq=1 << 28, n_tokens=0) == -4
    assert lib().csb_selective_scan(None, None, None) == -1 and lib().csb_last_error().startswith(b"csb_selective_scan")
    with pytest.raises(AssertionError):
        selective_scan(x, dt, A[:8], B, C)
    with pytest.raises(AssertionError):
        selective_scan(x.half(), dt, A, B, C)
    with pytest.raises(AssertionError):
        selective_scan(x, dt, A, B, C, state=torch.zeros(1, 16, 9, device="cuda"))
    with pytest.raises(CsbError, match="leading dimension"):
        selective_scan(x[:1].expand(12, 16), dt, A, B, C)
    torch.cuda.synchronize()


def test_refusals_of_the_workspace():
    x, dt, A, B, C, D, z, bias = (v.cuda() for v in inputs(22, 1024, 16, 1, 8, "f32"))
    out = torch.empty(1024, 16, device="cuda")
    args = csb_scan_args(type=0, channels=16, groups=1, n=8, n_seq=1, n_tokens=1024, d_x=x.data_ptr(), d_dt=dt.data_ptr(), d_B=B.data_ptr(), d_C=C.data_ptr(),
                         ldx=16, lddt=16, ldB=8, ldC=8, d_A=A.data_ptr(), d_out=out.data_ptr(), ldo=16)
    need = lib().csb_scan_workspace_bytes(args)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    assert need > 0
    assert lib().csb_selective_scan(args, None, None) == -1 and lib().csb_selective_scan(args, ws.data_ptr() + 8, None) == -1
    ws[need:] = 77
    assert lib().csb_selective_scan(args, ws.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert bool((ws[need:] == 77).all())
