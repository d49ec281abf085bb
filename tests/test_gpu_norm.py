"""Norms around a block (csb_block_norm) against their definition in 64 bits on the host, with bounds that follow the formulas
(layer_reference.norm)."""
import itertools
import math
import sys

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2005_05758_amd import block_norm
from paper_2005_05758_amd.binding import CsbError, csb_norm_args, csb_norm_operand, lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
types = pytest.mark.parametrize("fmt", sorted(TYPES))
SIZES = [(1, 1), (1, 64), (2, 7), (3, 8), (5, 65), (33, 128), (7, 130), (4, 512), (9, 515), (3, 2048), (2, 2053), (2, 4096), (3, 5003), (1, 8192), (2, 12001), (1, 32768)]


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def columns(x):
    """The same entries column by column, in a wider buffer: what a product leaves."""
    T, W = x.shape
    buffer = torch.full((W, T + -T % 4 + 4), math.nan, dtype=x.dtype, device=x.device)
    buffer[:, :T] = x.t()
    return buffer[:, :T].t()


def rows(x):
    buffer = torch.full((x.shape[0], x.shape[1] + 3), math.nan, dtype=x.dtype, device=x.device)
    buffer[:, 1:1 + x.shape[1]] = x
    return buffer[:, 1:1 + x.shape[1]]


def check(T, W, fmts="bf16", y=True, gate=False, x=True, after="rms", before="rms", weights=True, groups=1, gate_kind="silu", gate_first=False, scale=1.0,
          orders=(), seed=0, eps=1e-5, offset=0.0, change=None, in_place=None):
    """`fmts`: the type of all operands, or of y, gate, x, r and n.  `orders`: which of them lie column by column ("*": rows in a wider buffer)."""
    fmts = dict(zip("ygxrn", [fmts] * 5 if isinstance(fmts, str) else fmts))
    say(f"[norm] {T}x{W} {fmts} y={y} gate={gate} {gate_kind} {gate_first} x={x} {after}/{before} weights={weights} groups={groups} scale={scale} columns={orders}")
    t = torch.Generator().manual_seed(seed + T + W)
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    given = {"y": rnd(T, W) * 2 + offset if y else None, "g": rnd(T, W) * 2 if gate else None, "x": rnd(T, W) + offset if x else None}
    given = {k: v.to(TYPES[fmts[k]]) if v is not None else None for k, v in given.items()}
    factors = [1 + 0.3 * rnd(W), rnd(W), 0.5 + torch.rand(W, generator=t), 1 + 0.3 * rnd(W), rnd(W)] if weights else [None] * 5
    if change:
        change(given)

    def place(v, k):
        v = v.cuda()
        return columns(v) if k in orders else rows(v) if "*" in orders else v
    dev = {k: place(v, k) if v is not None else None for k, v in given.items()}
    out = place(torch.full((T, W), 7.0, dtype=TYPES[fmts["r"]]), "r") if in_place is None else dev[in_place]
    normed = place(torch.full((T, W), 7.0, dtype=TYPES[fmts["n"]]), "n") if before else None
    d = [f.cuda() if f is not None else None for f in factors]
    got = block_norm(dev["y"], gate=dev["g"], x=dev["x"], after=after, after_weight=d[0], after_bias=d[1], groups=groups, gate_kind=gate_kind,
                     gate_first=gate_first, scale=scale, scales=d[2], before=before, before_weight=d[3], before_bias=d[4], eps=eps, out=out, normed=normed)
    torch.cuda.synchronize()
    assert got[0] is out and got[1] is normed
    w = [ref.widen(f) if f is not None else None for f in factors]
    v = {k: ref.widen(v) if v is not None else None for k, v in given.items()}
    with np.errstate(all="ignore"):
        r, r_off, n, n_off = ref.norm(v["y"], v["g"], v["x"], after, w[0], w[1], groups, gate_kind == "sigmoid", gate_first, np.float32(scale), w[2], before,
                                      w[3], w[4], float(np.float32(eps)), "f32" if "f32" in (fmts["r"], fmts["n"] if before else fmts["r"]) else "bf16")
    if change is None:
        assert ref.within(ref.widen(out), r, r_off, fmts["r"]) <= 0
        assert n is None or ref.within(ref.widen(normed), n, n_off, fmts["n"]) <= 0
    return out, normed, r, n


@types
@pytest.mark.parametrize("T,W", SIZES)
def test_sizes(fmt, T, W):
    check(T, W, fmt)
    check(T, W, fmt, after="mean", before="mean", gate=True)
    check(T, W, fmt, orders="yn")


@pytest.mark.parametrize("T,W", [(1, 40), (5, 100), (8, 256), (9, 300), (17, 1030), (64, 513), (3, 3000), (12, 5000), (2, 9000), (3, 20000)])
@pytest.mark.parametrize("orders", ["y", "n", "ygxrn", "gr"])
def test_columns(T, W, orders):
    """Operands column by column and row by row in one call."""
    check(T, W, ["f32", "bf16", "f32", "bf16", "f16"], gate=True, orders=orders)


@pytest.mark.parametrize("x,columns,n", [("bf16", False, "bf16"), ("f16", False, "f16"), ("f32", False, "f32"), ("f32", False, "bf16"), ("f32", False, "f16"), ("f32", True, "f32"),
                                         ("f32", True, "bf16"), ("f32", True, "f16"), ("bf16", True, "bf16"), ("bf16", False, "f16")])
@pytest.mark.parametrize("T,W", [(1, 64), (3, 8200), (300, 96), (600, 1000), (1100, 256), (2100, 64), (5000, 24), (9, 32768), (130, 4096)])
def test_between_products(x, columns, n, T, W):
    """What a product leaves (binary32, column by column) and what the next one takes, the residual stream of either order."""
    orders = "yxrn" if columns else "yn"
    fmts = ["f32", "f32", x, x, n]
    check(T, W, fmts, orders=orders)
    if T < 1000:
        check(T, W, fmts, orders=orders, after="mean", before="mean", scale=0.3, weights=False)
        check(T, W, fmts, orders=orders, after=None, before="rms")
        check(T, W, fmts, orders=orders, after="rms", before=None, x=T > 100)


@pytest.mark.parametrize("after,before", itertools.product([None, "rms", "mean"], repeat=2))
@pytest.mark.parametrize("x", [True, False])
@pytest.mark.parametrize("orders", ["", "yn"])
def test_forms(after, before, x, orders):
    for gate, first, kind in ((False, False, "silu"), (True, False, "silu"), (True, True, "silu"), (True, False, "sigmoid"), (True, True, "sigmoid")):
        check(6, 200, "bf16", gate=gate, gate_first=first, gate_kind=kind, x=x, after=after, before=before, orders=orders, scale=0.7)
    check(6, 200, "f32", x=x, after=after, before=before, weights=False, orders=orders)


@types
@pytest.mark.parametrize("groups,width", [(2, 8), (16, 128), (8, 64), (3, 7), (5, 61), (4, 1), (2, 700), (3, 2500)])
@pytest.mark.parametrize("orders", ["", "r", "yg"])
def test_heads(fmt, groups, width, orders):
    check(19, groups * width, fmt, gate=True, x=False, before=None, groups=groups, orders=orders)
    check(5, groups * width, fmt, gate=True, gate_first=True, x=True, before=None, groups=groups, after="mean", orders=orders)


@types
def test_only_the_norm_before(fmt):
    x = torch.randn(9, 300, device="cuda").to(TYPES[fmt])
    r, n = block_norm(x=x, before="rms")
    again, m = block_norm(x=x, before="rms", out=torch.empty_like(x))
    torch.cuda.synchronize()
    assert r is x and torch.equal(n, m) and torch.equal(again, x)
    check(9, 300, fmt, y=False, after=None)


def test_types_of_operands():
    for fmts in itertools.product(["f32", "bf16"], ["f16"], ["f32", "bf16"], ["f32", "f16"], ["bf16", "f16"]):
        check(4, 96, list(fmts), gate=True)


@pytest.mark.parametrize("orders", ["", "*", "yxrn"])
@types
def test_in_place(fmt, orders):
    """The residual stream replaced where it is, and the block's output."""
    check(21, 333, fmt, orders=orders, in_place="x")
    check(21, 333, fmt, orders=orders, in_place="y")


@pytest.mark.parametrize("W", [64, 515, 5003])
def test_misaligned(W):
    for fmt in TYPES:
        check(11, W, fmt, gate=True, orders="*")


@pytest.mark.parametrize("orders", ["", "yn"])
def test_means_far_from_zero(orders):
    """Entries of a common size of 1000 times their spread: their variance keeps its digits (binary32 entries: those have the digits)."""
    check(5, 700, "f32", after="mean", before="mean", offset=1000.0, orders=orders)
    check(5, 700, "f32", x=False, after="mean", before=None, offset=-1e5, orders=orders)


@pytest.mark.parametrize("kind", ["rms", "mean"])
@pytest.mark.parametrize("size", [1e-30, 1e15, 1e25, 2e37])
def test_entries_of_any_size(kind, size):
    """Squares outside of binary32 do not matter."""
    def scaled(given):
        given["y"] *= size
    for orders in ("", "yr"):
        out, _, r, _ = check(4, 300, "f32", x=False, after=kind, before=None, weights=False, eps=0.0, orders=orders, change=scaled)
        assert np.isfinite(r).all() and np.abs(ref.widen(out) - r).max() <= 16 * ref.U * np.abs(r).max()


@pytest.mark.parametrize("orders", ["", "yxrn"])
def test_not_finite(orders):
    """A token with an entry that is not finite spoils itself and nothing else."""
    def spoil(given):
        given["y"][3, 5], given["x"][7, 199], given["y"][9, 0] = math.nan, math.inf, -math.inf
    out, normed, _, _ = check(12, 200, "bf16", change=spoil, orders=orders)
    clean, clean_n, _, _ = check(12, 200, "bf16", orders=orders)
    rest = [t for t in range(12) if t not in (3, 7, 9)]
    assert torch.equal(out[rest], clean[rest]) and torch.equal(normed[rest], clean_n[rest])
    assert not torch.isfinite(out[[3, 9]]).all() and not torch.isfinite(out[7, 199]) and not torch.isfinite(normed[[3, 7, 9]]).any(1).all()


def test_rows_of_zeros():
    for kind in ("rms", "mean"):
        r, n = block_norm(torch.zeros(3, 100, device="cuda"), after=kind, x=torch.zeros(3, 100, device="cuda"), before=kind, before_bias=torch.ones(100, device="cuda"))
        torch.cuda.synchronize()
        assert bool((r == 0).all()) and bool((n == 1).all())


@pytest.mark.parametrize("orders", ["", "n"])
def test_what_lies_behind_the_tokens_stays(orders):
    x = torch.randn(5, 40, device="cuda")
    buffer = torch.full((40, 8), 3.0, device="cuda") if orders else torch.full((8, 45), 3.0, device="cuda")
    view = buffer[:, :5].t() if orders else buffer[:5, :40]
    block_norm(x=x, before="rms", normed=view)
    torch.cuda.synchronize()
    assert bool((buffer[:, 5:] == 3.0).all()) if orders else bool((buffer[5:] == 3.0).all() and (buffer[:, 40:] == 3.0).all())


def test_entries_past_32_bits():
    """More than 2^31 entries, row by row and column by column."""
    ld = 2 ** 25
    buffer = torch.empty(70 * ld, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(70, 96, device="cuda").bfloat16()
    view = buffer.as_strided((70, 96), (ld, 1))
    view.copy_(x)
    a, b = block_norm(x=view, before="rms")[1], block_norm(x=x, before="rms")[1]
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    wide = torch.randn(50, 70, device="cuda").bfloat16()
    turned = buffer.as_strided((50, 70), (1, ld))
    turned.copy_(wide)
    a, b = block_norm(x=turned, before="rms")[1], block_norm(x=wide, before="rms")[1]
    torch.cuda.synchronize()
    assert (a.float() - b.float()).abs().max() <= 2 ** -7 * b.float().abs().max()          # (sums in another order)


@pytest.mark.parametrize("orders", ["", "yn"])
def test_stream_and_graph(orders):
    y, x = torch.randn(70, 300, device="cuda"), torch.randn(70, 300, device="cuda").bfloat16()
    if orders:
        y = columns(y)
    normed = columns(torch.zeros_like(x)) if orders else torch.zeros_like(x)

    def once(stream=None):
        torch.cuda.synchronize()
        got = [t.clone() for t in block_norm(y, x=x, after="rms", before="rms", normed=normed, out=torch.empty_like(x), stream=stream)]
        torch.cuda.synchronize()
        return got
    want = once()
    for got in (once(), once(torch.cuda.Stream())):
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(x)
    with torch.cuda.graph(graph):
        block_norm(y, x=x, after="rms", before="rms", out=out, normed=normed)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        want = once()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(normed, want[1])


def test_refusals():
    y, x, out, n = (torch.zeros(12, 16, device="cuda") for _ in range(4))
    op = lambda t, **kw: csb_norm_operand(**{**dict(d=t.data_ptr(), ld=16, type=0, columns=0), **kw})     # noqa: E731
    good = dict(n_tokens=12, width=16, groups=1, after=1, before=1, scale=1.0, eps=1e-5, y=op(y), x=op(x), r=op(out), out=op(n))

    def call(**change):
        return lib().csb_block_norm(csb_norm_args(**{**good, **change}), None)
    none = csb_norm_operand()
    assert call() == 0 and call(n_tokens=0) == 0 and call(r=none) == 0 and call(x=none) == 0 and call(before=0, out=none) == 0
    assert call(y=op(y, ld=12, columns=1)) == 0
    for change in (dict(n_tokens=-1), dict(width=0), dict(groups=0), dict(groups=3), dict(after=3), dict(before=-1), dict(gate_kind=2), dict(eps=-1.0), dict(eps=math.nan),
                   dict(y=none, x=none), dict(y=none), dict(y=none, after=0, gate=op(y)), dict(out=none), dict(before=0, r=none), dict(out=op(out)),
                   dict(y=op(y, ld=15)), dict(y=op(y, ld=11, columns=1)), dict(x=op(x, type=3)), dict(r=op(out, ld=0)), dict(y=op(y, d=y.data_ptr() + 2)),
                   dict(d_after_w=y.data_ptr() + 2)):
        assert call(**change) == -1, change
    assert call(width=32769, y=op(y, ld=32769), x=none, r=op(out, ld=32769), out=op(n, ld=32769), groups=1) == -4
    assert call(groups=2) == -4
    assert call(n_tokens=1 << 40) == -4
    assert lib().csb_block_norm(None, None) == -1 and lib().csb_last_error().startswith(b"csb_block_norm")
    for bad in (dict(after="l2"), dict(after_weight=torch.ones(15, device="cuda")), dict(after_weight=torch.ones(16, device="cuda").half()),
                dict(out=torch.empty(12, 15, device="cuda")), dict(normed=torch.empty(12, 16, device="cuda")), dict(x=x[:6])):
        with pytest.raises((AssertionError, KeyError)):
            block_norm(y, **bad)
    with pytest.raises(CsbError, match="leading dimension"):
        block_norm(y[:1].expand(12, 16), after="rms")
    with pytest.raises(AssertionError, match="contiguous"):
        block_norm(torch.zeros(12, 32, device="cuda")[:, ::2], after="rms")
    torch.cuda.synchronize()
