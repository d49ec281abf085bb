"""A model of the chunk-by-chunk form of the delta rule in which every operand of a product keeps a given number of
bfloat16 parts (test infrastructure): what a kernel that kept fewer of them would return."""
import numpy as np
import torch

OPERANDS = ("S", "R", "U", "M", "P")


def kept(x, parts):
    """x in binary32, as the sum of its first `parts` bfloat16 parts."""
    rest = torch.from_numpy(np.asarray(x, np.float64)).float()
    total = np.zeros(rest.shape)
    for _ in range(parts):
        near = rest.bfloat16().float()
        total += near.double().numpy()
        rest = rest - near
    return total


def chunked(q, k, v, g, beta, scale, S, parts=None, chunk=64):
    """One sequence: q, k [tokens, heads_k, dk], v [tokens, heads_v, dv], g, beta [tokens, heads_v], S [heads_v, dk, dv], all
    float64.  parts: {operand: bfloat16 parts}, 3 where it is not named.  Returns (out, S)."""
    n = {**dict.fromkeys(OPERANDS, 3), **(parts or {})}
    T, HV, DV = v.shape
    out, S = np.empty((T, HV, DV)), S.copy()
    for h in range(HV):
        kh = h // (HV // k.shape[1])
        for c in range(0, T, chunk):
            K, Q, V, b = k[c:c + chunk, kh], q[c:c + chunk, kh], v[c:c + chunk, h], beta[c:c + chunk, h]
            G = np.cumsum(g[c:c + chunk, h])
            low = np.tril(np.exp(np.minimum(G[:, None] - G[None, :], 0.0)))
            M = np.linalg.inv(np.eye(len(G)) + np.tril(b[:, None] * low * (K @ K.T), -1)) * b[None, :]
            Sp, grow = kept(S[h], n["S"]), np.exp(G)[:, None]
            R = V - grow * (K @ Sp)
            U = kept(M, n["M"]) @ kept(R, n["R"])
            out[c:c + chunk, h] = scale * (grow * (Q @ Sp) + kept(low * (Q @ K.T), n["P"]) @ kept(U, n["U"]))
            S[h] = (np.exp(G[-1]) * S[h] + K.T @ kept(np.exp(G[-1] - G)[:, None] * U, n["U"])).astype(np.float32)
    return out, S
