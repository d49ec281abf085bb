"""The operators around a recurrent layer from their definitions, in 64 bits on the host, with what rounding may add to each
result (test infrastructure).

U = 2^-24 is half a unit in the last place of binary32.  The bounds follow the sums as they are formed: a sum of n terms in any order is
off by at most n U of its terms' absolute values, a product by U, the card's exponential of a binary32 number by 2 U, its reciprocal by 2 U."""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit in the last place, of the value
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}   # numbers below the normal ones


def widen(t):
    """A torch tensor of any float type as float64 numbers (every value of the types is one)."""
    return t.detach().cpu().double().numpy()


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def silu(x):
    return x * sigmoid(x)


def gate_off(fmt, x):
    """What SiLU is off of its value: the exponential 4 U (argument and all), sum, reciprocal and product 4 U more; where it is rounded to 16 bits afterwards its
    argument x log2 e is two numbers' rounded product, U of |x| log2 e of ln 2 each: 1 + 1/4 |x| U (log2 e's own rounding is below U / 4)."""
    return (8 + (0.0 if fmt == "f32" else 1.25) * np.abs(x)) * U


def conv(x, w, b, act, ranges, slots, state, fmt):
    """x [T, C], w [C, W], state [n, W - 1, C].  Returns (out, off, state): out is NaN where no sequence has a token."""
    T, C = x.shape
    W = w.shape[1]
    out, off, state = np.full((T, C), np.nan), np.zeros((T, C)), state.copy()
    for (first, end), s in zip(ranges, slots):
        v = np.concatenate([state[s] if s >= 0 else np.zeros((W - 1, C)), x[first:end]])
        n = end - first
        y = b + sum(v[j:j + n] * w[:, j] for j in range(W))
        size = np.abs(b) + sum(np.abs(v[j:j + n] * w[:, j]) for j in range(W))
        out[first:end] = silu(y) if act else y
        # the sum: W + 1 roundings.  SiLU's slope is at most 1.1
        off[first:end] = 1.1 * (W + 1) * U * size + gate_off(fmt, y) * np.abs(out[first:end])
        if s >= 0 and W > 1:
            state[s] = v[n:]
    return out, off, state


def scan(x, dt, A, B, C, D, z, bias, softplus, ranges, slots, state, fmt):
    """x, dt, z [T, ch], B, C [T, G, n], A [ch, n], state [S, ch, n].  Returns (out, off, state, state_off)."""
    T, ch = x.shape
    G, n = B.shape[1:]
    out, off = np.full((T, ch), np.nan), np.zeros((T, ch))
    state, soff = state.copy(), np.zeros(state.shape)
    step = dt + bias
    # dt + bias: U of it; ln(1 + e^s) has a slope of at most 1 and 12 U of its own (exponential 4, quotient 4, series and sum 4).  From 16 bits the
    # exponential's argument is two numbers' rounded product: e^-|s| is 1.25 |s| U more off, and ln(1 + e) that times e / (1 + e) <= ln(1 + e)
    step_off = U * np.abs(step)
    if softplus:
        with np.errstate(invalid="ignore"):
            short = 0.0 if fmt == "f32" else np.where(np.abs(step) < 1000, 1.25 * np.abs(step) * np.log1p(np.exp(-np.abs(step))), 0.0) * U
        step = np.maximum(step, 0.0) + np.log1p(np.exp(-np.abs(step)))
        slope = -np.expm1(-step)
        step_off = slope * step_off + 12 * U * step + short
    gate = silu(z) if z is not None else np.ones((T, ch))
    for (first, end), s in zip(ranges, slots):
        h = state[s].copy() if s >= 0 else np.zeros((ch, n))
        size, e = np.abs(h), np.zeros((ch, n))
        for t in range(first, end):
            b, c = (np.repeat(m[t], ch // G, axis=0) for m in (B, C))
            arg = step[t][:, None] * A
            a = np.exp(arg)
            # the argument: A log2 e and the product rounded, the step's error; over chunks the sum of the steps may be 40 U off; then the exponential
            # and the fused product and sum
            arg_off = step_off[t][:, None] * np.abs(A) + 43 * U * np.abs(arg)
            into = step[t][:, None] * x[t][:, None] * b
            into_off = (step_off[t] * np.abs(x[t]))[:, None] * np.abs(b) + 3 * U * np.abs(into)
            e = a * e + (arg_off + 4 * U) * a * size + into_off
            h, size = a * h + into, a * size + np.abs(into)
            y = (c * h).sum(1) + D * x[t]
            y_off = (np.abs(c) * e).sum(1) + (n + 3) * U * ((np.abs(c) * size).sum(1) + np.abs(D * x[t]))
            out[t] = y * gate[t]
            off[t] = np.abs(gate[t]) * (1.001 * y_off + (U + (gate_off(fmt, z[t]) if z is not None else 0.0)) * np.abs(y))
        if s >= 0:
            state[s], soff[s] = h, 1.001 * e
    return out, off, state, soff


def within(got, want, off, fmt):
    """How far entries are outside of what they may be, the type's rounding included (not above 0: fine)."""
    there = ~np.isnan(want)
    if not there.any():
        return 0.0
    allowed = off[there] + HALF[fmt] * (np.abs(want[there]) + off[there]) + TINY[fmt]
    return float((np.abs(got[there] - want[there]) - allowed).max())


def norm(y, gate, x, after, aw, ab, groups, sigmoid_gate, gate_first, scale, s, before, bw, bb, eps, fmt):
    """All [T, W] or None (weights [W]); fmt: "f32" where one of the results is.  Returns (r, off, n, off): n None without a norm before."""
    T, W = (x if x is not None else y).shape

    def unit(v, e, kind, w, b, parts):
        """norm(v) of entries that are off by e, and how far its own are: v - m is off by e's and the mean's, the factor by what its
        root of a mean square is, 2 U of its own; the product, w and b 4 U more."""
        if not kind:
            return v, e
        v, e = v.reshape(T, parts, -1), e.reshape(T, parts, -1)
        if kind == "mean":
            v, e = v - v.mean(-1, keepdims=True), e + e.mean(-1, keepdims=True) + U * np.abs(v - v.mean(-1, keepdims=True))
        ms = (v * v).mean(-1, keepdims=True) + eps
        f = 1.0 / np.sqrt(ms)
        f_off = f * ((np.abs(v) * e).mean(-1, keepdims=True) / ms + 3 * U)
        out = (v * f).reshape(T, W)
        off = (e * f + np.abs(v) * f_off).reshape(T, W) + 2 * U * np.abs(out)
        w, b = w if w is not None else np.ones(W), b if b is not None else np.zeros(W)
        return out * w + b, off * np.abs(w) + 2 * U * (np.abs(out * w) + np.abs(b))
    r, off = np.zeros((T, W)), np.zeros((T, W))
    if y is not None:
        r = y.copy()
        act = None
        if gate is not None:
            act = sigmoid(gate) if sigmoid_gate else silu(gate)
        if act is not None and gate_first:
            r, off = r * act, (U + gate_off(fmt, gate)) * np.abs(r * act)
        r, off = unit(r, off, after, aw, ab, groups)
        if act is not None and not gate_first:
            r, off = r * act, off * np.abs(act) + (U + gate_off(fmt, gate)) * np.abs(r * act)
        m = scale * (s if s is not None else np.ones(W))
        r, off = r * m, (off + 3 * U * np.abs(r)) * np.abs(m)
    if x is not None:
        r = r + x
        off = off + U * np.abs(r)
    off = 1.001 * off
    if not before:
        return r, off, None, None
    n, n_off = unit(r, off, before, bw, bb, 1)
    return r, off, n, 1.001 * n_off


UNITS = 2.0 ** 38


def sample(s, T, k, p, q, r):
    """One row s of float64 logits (values of the type); T, k, p, q, r numbers of the types that they are given in.  Returns (token, weights that are kept)."""
    s = np.where(np.isnan(s), -np.inf, s)
    V, m = len(s), s.max()
    kept = np.zeros(V, np.int64)
    if m == -np.inf:
        return -1, kept
    order = np.lexsort((np.arange(V), -s))
    w = np.zeros(V, np.int64)
    if T > 0:
        with np.errstate(all="ignore"):
            d = (s - m) / T
            w = np.where(s == m, UNITS, np.where(d > -40, np.floor(np.exp(d) * UNITS), 0.0)).astype(np.int64)
    else:
        w[order[0]] = int(UNITS)
    keep = order
    if 0 < k < V:
        keep = keep[:k]
    if p < 1:
        units = [int(u) for u in w[keep]]
        limit, before, n = sum(units) * int(max(p, 0.0) * 2 ** 24) >> 24, 0, 0
        while n < len(units) and (before < limit or n == 0):
            before += units[n]
            n += 1
        keep = keep[:n]
    if q > 0:
        keep = keep[w[keep] >= int(min(q, 1.0) * UNITS)]
    kept[keep] = w[keep]
    total = int(kept.sum())
    limit = total * min(int(max(r, 0.0) * 2 ** 24), 2 ** 24 - 1) >> 24
    return int(np.searchsorted(np.cumsum(kept), limit, side="right")), kept
