"""The language-model operators from their definitions, in 64 bits on the host (test infrastructure): the
gated delta rule token by token, adapters column by column, verification in whole numbers."""
import numpy as np


def widen(t):
    """A torch tensor of any float type as float64 numbers (every value of the types is one)."""
    return t.detach().cpu().double().numpy()


def delta(q, k, v, g, beta, scale, ranges, slots, state, touched=None):
    """ranges: (first, end) of each sequence; slots: its state or -1.  Returns (out, state); out is NaN where
    no sequence has a token."""
    T, HV, DV = v.shape
    HK, DK = q.shape[1:]
    out = np.full((T, HV, DV), np.nan)
    state = state.copy()
    for (first, end), s in zip(ranges, slots):
        for h in range(HV):
            kh = h // (HV // HK)
            S = state[s, h].copy() if s >= 0 else np.zeros((DK, DV))
            for t in range(first, end):
                S = np.exp(g[t, h]) * S
                u = beta[t, h] * (v[t, h] - S.T @ k[t, kh])
                S = S + np.outer(k[t, kh], u)
                out[t, h] = scale * (S.T @ q[t, kh])
            if s >= 0:
                state[s, h] = S
    return out, state


def adapters(Y, X, A, B, ranges, ids, scales, ranks):
    Y = Y.copy()
    for (first, end), a in zip(ranges, ids):
        if 0 <= a < A.shape[0]:
            r = min(max(int(ranks[a]), 0), A.shape[1])
            Y[:, first:end] += scales[a] * (B[a][:, :r] @ (A[a][:r] @ X[:, first:end]))
    return Y


def adapter_sizes(Y, X, A, B, ranges, ids, scales, ranks):
    """The same sums over absolute values: what rounding errors are measured by."""
    return adapters(np.abs(Y), np.abs(X), np.abs(A), np.abs(B), ranges, ids, np.abs(scales), ranks)


def units(w):
    with np.errstate(invalid="ignore"):
        w = np.where(w > 0, np.minimum(w, np.float32(1.0)), np.float32(0.0))
    return (w.astype(np.float64) * 2.0 ** 38).astype(np.int64)


def verify(p, q, drafts, u, r, counts):
    """p [N, K+1, V], q [N, K, V] or None: float32 values.  Returns (tokens, accepted)."""
    N, K1, V = p.shape
    tokens, accepted = np.full((N, K1), -1, np.int32), np.zeros(N, np.int32)
    for b in range(N):
        n, count = 0, min(max(int(counts[b]), 0), K1 - 1)
        while n < count:
            d = int(drafts[b, n])
            if not 0 <= d < V or not np.float32(u[b, n]) * (q[b, n, d] if q is not None else np.float32(1)) < p[b, n, d]:
                break
            tokens[b, n] = d
            n += 1
        accepted[b] = n
        left = p[b, n].copy()
        if n < count and q is not None:
            with np.errstate(invalid="ignore"):
                left = p[b, n] - q[b, n]
        elif n < count and 0 <= drafts[b, n] < V:
            left[drafts[b, n]] -= np.float32(1)
        m = min(int(max(float(r[b]), 0.0) * 2 ** 24), 2 ** 24 - 1)
        for w in (units(left), units(p[b, n])):
            cum = np.cumsum(w)
            total = int(cum[-1])
            if total > 0:
                tokens[b, n] = int(np.searchsorted(cum, total * m >> 24, side="right"))
                break
    return tokens, accepted
