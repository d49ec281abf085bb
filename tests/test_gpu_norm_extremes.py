"""Norms of entries that are not finite, or far outside of the others' size: what the definition gives for the other entries of their token, and the same bits for
every other token."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2005_05758_amd import block_norm
from test_gpu_norm import TYPES, columns

pytestmark = pytest.mark.gpu

# rows by 8, 16, 64, 256 and 1024 lanes, in registers and read again; tokens side by side, and what stands between products
FORMS = [("rows", 64), ("rows", 61), ("rows", 128), ("rows", 200), ("rows", 2053), ("rows", 5003), ("rows", 8200), ("rows", 20000), ("columns", 200), ("columns", 515),
         ("columns", 20001), ("products", 96), ("products", 4104)]
forms = pytest.mark.parametrize("form,W", FORMS)
T = 24


def operands(form, W, fmt, seed=0, tokens=T):
    t = torch.Generator().manual_seed(seed + W)
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    y = rnd(tokens, W).to(torch.float32 if form == "products" else TYPES[fmt])
    return y, rnd(tokens, W).to(TYPES[fmt]), [1 + 0.3 * rnd(W), rnd(W), 0.5 + torch.rand(W, generator=t), 1 + 0.3 * rnd(W), rnd(W)]


def run(form, y, x, factors, after, before):
    y, x, f = y.cuda(), x.cuda(), [v.cuda() for v in factors]
    r, n = torch.empty_like(x), torch.empty_like(x)
    if form != "rows":
        y, n = columns(y), columns(n)
    if form == "columns":
        x, r = columns(x), columns(r)
    print(f"[norm] {form} {y.shape[0]}x{y.shape[1]} {x.dtype} {after}/{before}", flush=True)
    block_norm(y, x=x, after=after, after_weight=f[0], after_bias=f[1], scale=0.7, scales=f[2], before=before, before_weight=f[3], before_bias=f[4], out=r, normed=n)
    torch.cuda.synchronize()
    return r, n


def agrees(got, want, size, fmt, roundings):
    """The same entries NaN, the same infinite, the others within so many roundings of `size`."""
    got = ref.widen(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    there = np.isfinite(want)
    allowed = ref.HALF[fmt] * np.abs(want[there]) + roundings * 1.001 * ref.U * size[there] + ref.TINY[fmt]
    assert (np.abs(got[there] - want[there]) <= allowed).all()


@pytest.mark.parametrize("fmt", sorted(TYPES))
@forms
def test_infinite_entries_of_a_mean_square(form, W, fmt):
    """Of a token with infinite entries: those are NaN (infinity over infinity), its others zero before weight and bias are applied."""
    y, x, factors = operands(form, W, fmt)
    y[3, W // 2], y[9, 0], x[14, W - 1], y[20, 1], y[20, W - 2] = math.inf, -math.inf, math.inf, math.inf, -math.inf
    r, n = run(form, y, x, factors, "rms", "rms")
    aw, ab, s, bw, bb = (ref.widen(f) for f in factors)
    wide, scale = ref.widen(x), float(np.float32(0.7))
    with np.errstate(all="ignore"):
        want, _, want_n, _ = ref.norm(ref.widen(y), None, wide, "rms", aw, ab, 1, False, False, scale, s, "rms", bw, bb, float(np.float32(1e-5)), fmt)
    hit = [3, 9, 20]                                     # r: x + scale s (0 aw + ab); scale s, its product with ab, the sum
    assert np.isnan(want[hit]).sum() == 4 and np.isnan(want_n[hit]).all()
    agrees(r[hit], want[hit], (np.abs(wide) + np.abs(scale * s * ab))[hit], fmt, 3)
    agrees(n[hit], want_n[hit], np.zeros((3, W)), fmt, 0)
    assert np.isnan(want_n[14]).sum() == 1 and np.isinf(want[14, W - 1])
    agrees(n[14], want_n[14], np.abs(bb), fmt, 0)        # 0 bw + bb


@pytest.mark.parametrize("fmt", sorted(TYPES))
@forms
def test_nan_and_a_mean_square(form, W, fmt):
    y, x, factors = operands(form, W, fmt)
    y[3, W // 2], x[14, W - 1] = math.nan, math.nan
    r, n = run(form, y, x, factors, "rms", "rms")
    assert bool(torch.isnan(r[3]).all()) and bool(torch.isnan(n[[3, 14]]).all()) and int(torch.isnan(r[14]).sum()) == 1
    rest = [t for t in range(T) if t not in (3, 14)]
    assert bool(torch.isfinite(r[rest]).all()) and bool(torch.isfinite(n[rest]).all())


@pytest.mark.parametrize("fmt", sorted(TYPES))
@forms
def test_entries_that_are_not_finite_and_a_mean(form, W, fmt):
    """A token whose mean is not finite has no norm: all of its entries are NaN, wherever the one that spoils it lies."""
    for value in (math.inf, -math.inf, math.nan):
        y, x, factors = operands(form, W, fmt)
        y[3, W // 2], y[9, 0], x[14, W - 1], x[17, 0], y[20, 1], y[20, W - 2] = value, value, value, value, value, -value
        r, n = run(form, y, x, factors, "mean", "mean")
        assert bool(torch.isnan(r[[3, 9, 20]]).all()) and bool(torch.isnan(n[[3, 9, 14, 17, 20]]).all())
        rest = [t for t in range(T) if t not in (3, 9, 14, 17, 20)]
        assert bool(torch.isfinite(r[rest]).all()) and bool(torch.isfinite(n[rest]).all())


@forms
@pytest.mark.parametrize("kind", ["rms", "mean"])
def test_other_tokens_keep_their_bits(form, W, kind):
    """Next to tokens with infinities, NaN, entries whose squares leave binary32, and entries that are all but nothing."""
    y, x, factors = operands(form, W, "f32", seed=1, tokens=600)       # (more tokens side by side in a wavefront than of 24)
    clean = run(form, y, x, factors, kind, kind)
    values = [math.inf, math.nan, 1e25, 1e-25, -math.inf, 3e38, 1e-38]
    spoiled = list(range(3, 600, 19))
    for t in spoiled:
        y[t], x[t] = values[t % 7], -values[t % 7]
    got = run(form, y, x, factors, kind, kind)
    rest = [t for t in range(600) if t not in spoiled]
    for a, b in zip(got, clean):
        assert torch.equal(a[rest], b[rest])
