"""The measured cases of the language-model operators: gated delta rule, adapters, draft verification.

A case is a dict of plain values.  `kind` picks the operator:

  "chunked"    delta_chunked: the gated delta rule over whole prompts, packed one behind the other
  "recurrent"  delta_recurrent: the same rule for the few tokens of a decoding step, states in a pool
  "adapter"    adapter_add: low-rank adapters of many requests added to a shared projection's result
  "verify"     verify_drafts: drafted tokens against the target's probabilities, from given numbers

run() computes a case in its plain form, elementary torch operations in 32 bits; with `own` set it makes
the framework's calls.  exact() computes it from the definition in 64 bits, token by token.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
CHUNK = 64                   # tokens that the plain form of the delta rule takes at once
UNITS = 2.0 ** 38            # verification: probabilities are counted in whole units of 2^-38


def _delta(name, kind, seqs, tokens, heads_k, heads_v, dk, dv, fmt, spread):
    """`tokens`: all sequences together.  `spread`: longest over mean length (1: all alike)."""
    return {"name": name, "kind": kind, "seqs": seqs, "tokens": tokens, "heads_k": heads_k, "heads_v": heads_v,
            "dk": dk, "dv": dv, "format": fmt, "spread": spread}


def _adapter(name, rows, cols, batch, segments, adapters, rank, fmt):
    return {"name": name, "kind": "adapter", "rows": rows, "cols": cols, "batch": batch, "segments": segments,
            "adapters": adapters, "rank": rank, "format": fmt}


def _verify(name, requests, drafts, vocab, fmt, draft_probs):
    return {"name": name, "kind": "verify", "requests": requests, "drafts": drafts, "vocab": vocab, "format": fmt,
            "draft_probs": draft_probs}


def listed():
    return [
        # One long document read at once: few heads, hundreds of dependent chunks.
        _delta("chunked_long_bf16", "chunked", 1, 32768, 8, 16, 128, 128, "bf16", 1.0),
        # The prompts of many requests as a server packs them, of very different lengths.
        _delta("chunked_packed_bf16", "chunked", 48, 16411, 16, 16, 128, 128, "bf16", 4.0),
        # Full precision and widths that fill no tile, as a small research model has them.
        _delta("chunked_odd_f32", "chunked", 5, 1999, 2, 6, 96, 80, "f32", 2.0),
        # One utterance of 100 frames through a small layer: a call of two chunks.
        _delta("chunked_short_f16", "chunked", 1, 100, 4, 4, 64, 64, "f16", 1.0),
        # One request, one token: the smallest call, where latency is all there is.
        _delta("recurrent_one_bf16", "recurrent", 1, 1, 8, 16, 128, 128, "bf16", 1.0),
        # A full batch of requests, one token each.
        _delta("recurrent_batch_bf16", "recurrent", 64, 64, 16, 32, 128, 128, "bf16", 1.0),
        # Requests that bring a few drafted tokens each, an odd batch of them.
        _delta("recurrent_drafts_f16", "recurrent", 33, 131, 8, 16, 128, 128, "f16", 2.0),
        # Decoding: 64 requests of one token each, most with an adapter of their own.
        _adapter("adapter_decode_bf16", 4096, 4096, 64, 64, 48, 16, "bf16"),
        # Prompts of nine requests beside the large square projection, ranks mixed.
        _adapter("adapter_prefill_bf16", 8192, 8192, 2048, 9, 6, 64, "bf16"),
        # The frames of one utterance and an odd input, in full precision.
        _adapter("adapter_odd_f32", 2048, 665, 99, 3, 2, 8, "f32"),
        # One request, a vocabulary of odd size, drafts from a smaller model.
        _verify("verify_one_f32", 1, 4, 20011, "f32", True),
        # A batch and a large vocabulary.
        _verify("verify_batch_f32", 64, 7, 131071, "f32", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunked", "chunked", "recurrent", "recurrent", "adapter", "adapter", "verify"])
    if kind in ("chunked", "recurrent"):
        hk = rng.choice([1, 2, 4, 8])
        hv = hk * rng.choice([1, 2, 3] if hk < 8 else [1, 2])
        fmt = rng.choice(["bf16", "bf16", "f16", "f32"])
        dk, dv = (rng.choice([64, 128, _log(rng, 16, 128), _log(rng, 16, 256)]) for _ in range(2))
        if kind == "chunked":
            tokens = _log(rng, 33, 16384)
            seqs = min(_log(rng, 1, 32), max(1, tokens // 8))
        else:
            seqs = _log(rng, 1, 96)
            tokens = seqs if rng.random() < 0.5 else _log(rng, seqs, 6 * seqs)
        c = _delta("", kind, seqs, tokens, hk, hv, dk, dv, fmt, round(rng.uniform(1.0, 4.0), 1))
    elif kind == "adapter":
        batch = _log(rng, 1, 2048)
        segments = min(batch, _log(rng, 1, 64))
        c = _adapter("", _log(rng, 512, 8192), _log(rng, 153, 8192), batch, segments, rng.randint(1, segments),
                     rng.choice([4, 8, 16, 32, 64, rng.randint(1, 64)]), rng.choice(["bf16", "bf16", "f16", "f32"]))
    else:
        c = _verify("", _log(rng, 1, 64), rng.randint(1, 8), _log(rng, 500, 131072), rng.choice(["f32", "f32", "f16", "bf16"]),
                    rng.random() < 0.7)
    del c["name"]
    return c


def _lengths(seed, n, total, spread):
    """n lengths of `total` together, none of them zero, the longest about spread * mean."""
    g = np.random.Generator(np.random.PCG64(seed))
    w = np.exp(g.uniform(-math.log(spread), 0.0, n)) if spread > 1.0 else np.ones(n)
    cut = np.floor(np.cumsum(w) / w.sum() * (total - n) + 0.5).astype(np.int64)
    return np.diff(np.concatenate([[0], cut])) + 1


def _starts(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()


def prepare(case, seed):
    t = torch.Generator(device="cuda").manual_seed(seed + 104729)

    def normal(*shape):
        return torch.randn(shape, generator=t, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=t, device="cuda")

    kind, typ = case["kind"], TYPES[case["format"]]
    if kind in ("chunked", "recurrent"):
        N, T, HK, HV, DK, DV = (case[k] for k in ("seqs", "tokens", "heads_k", "heads_v", "dk", "dv"))
        lengths = _lengths(seed, N, T, case["spread"])

        def unit(x):                                         # what a layer hands over: SiLU, then length one
            return torch.nn.functional.normalize(x * torch.sigmoid(x), dim=-1)
        decay = 1.0 + 15.0 * uniform(HV)                     # of a head; the step sizes are a token's
        step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(T, HV))
        pool = N + 3                                         # requests sit anywhere in the pool of states
        return {"case": case, "q": unit(normal(T, HK, DK)).to(typ), "k": unit(normal(T, HK, DK)).to(typ),
                "v": normal(T, HV, DV).to(typ), "g": -decay * step, "beta": torch.sigmoid(normal(T, HV)),
                "starts": _starts(lengths), "longest": int(lengths.max()),
                "slots": torch.randperm(pool, generator=t, device="cuda")[:N].to(torch.int32),
                "state": 0.3 * normal(pool, HV, DK, DV), "scale": DK ** -0.5}
    if kind == "adapter":
        n, segs, R = case["batch"], case["segments"], case["rank"]
        lengths = _lengths(seed, segs, n, 3.0 if segs < n else 1.0)
        ids = torch.randint(0, case["adapters"], (segs,), generator=t, device="cuda")
        if segs == case["adapters"] or segs == n:            # a request of its own each, as far as they go
            ids = torch.arange(segs, device="cuda") % case["adapters"]
        if segs > 2:
            ids[1] = -1                                      # one request in every batch has none
        ranks = torch.randint((R + 1) // 2, R + 1, (case["adapters"],), generator=t, device="cuda")
        ranks[0] = R
        return {"case": case, "X": normal(case["cols"], n).to(typ), "Y": normal(case["rows"], n),
                "A": (normal(case["adapters"], R, case["cols"]) * case["cols"] ** -0.5).to(typ),
                "B": (normal(case["adapters"], case["rows"], R) * 0.05).to(typ),
                "ids": ids.to(torch.int32), "starts": _starts(lengths), "longest": int(lengths.max()),
                "ranks": ranks.to(torch.int32), "scales": 16.0 / ranks.float()}
    B, K, V = case["requests"], case["drafts"], case["vocab"]
    logits = 2.5 * normal(B, K + 1, V)
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits[:, :K] + 0.7 * normal(B, K, V), -1)
    drafts = torch.multinomial(q.reshape(B * K, V), 1, generator=t).view(B, K)
    counts = torch.randint((K + 1) // 2, K + 1, (B,), generator=t, device="cuda")
    return {"case": case, "p": p.to(typ), "q": q.to(typ) if case["draft_probs"] else None, "drafts": drafts.to(torch.int32),
            "counts": counts.to(torch.int32), "u": uniform(B, K), "r": uniform(B)}


def _padded(st):
    """Token numbers [sequences, longest] of packed sequences, and which of them are tokens."""
    first, end = st["starts"][:-1, None].long(), st["starts"][1:, None].long()
    at = first + torch.arange(st["longest"], device="cuda")
    there = at < end
    return torch.where(there, at, torch.zeros_like(at)), there


def _delta_inputs(st, steps, dtype):
    """q, k, v, decay and beta by sequence and head, [N, HV, steps, ...]; places that are no token change nothing."""
    at, there = _padded(st)
    pad = steps - at.shape[1]
    at = torch.nn.functional.pad(at, (0, pad))
    there = torch.nn.functional.pad(there, (0, pad))
    group = st["v"].shape[1] // st["q"].shape[1]

    def by_head(x, rep=1):
        return x[at].to(dtype).repeat_interleave(rep, 2).transpose(1, 2)
    live = there[:, None, :].to(dtype)
    return (at, there, by_head(st["q"], group), by_head(st["k"], group), by_head(st["v"]),
            by_head(st["g"]) * live, by_head(st["beta"]) * live)


def _chunked_plain(st):
    chunks = -(-st["longest"] // CHUNK)
    at, there, q, k, v, g, b = _delta_inputs(st, chunks * CHUNK, torch.float32)
    N, HV = v.shape[:2]
    q, k, v = (x.reshape(N, HV, chunks, CHUNK, -1) for x in (q, k, v))
    g, b = (x.reshape(N, HV, chunks, CHUNK) for x in (g, b))
    G = torch.cumsum(g, -1)                                  # decay from the chunk's start, as a logarithm
    low = torch.tril(torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda"))
    between = torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], torch.full_like(G[..., :, None], -math.inf)))
    T = torch.matmul(k, k.transpose(-1, -2)) * between * b[..., None] * torch.tril(torch.ones_like(between[0, 0, 0]), -1)
    inv = torch.eye(CHUNK, device="cuda").repeat(N, HV, chunks, 1, 1)
    for i in range(1, CHUNK):                                # (1 + T)^-1 by forward substitution, all chunks at once
        inv[..., i, :] -= torch.matmul(T[..., i:i + 1, :i], inv[..., :i, :])[..., 0, :]
    P = torch.matmul(q, k.transpose(-1, -2)) * between
    S = st["state"][st["slots"].long()]
    out = torch.empty_like(v)
    for c in range(chunks):                                  # each chunk from the state of the one before
        grow = torch.exp(G[:, :, c])[..., None]
        u = torch.matmul(inv[:, :, c], b[:, :, c, :, None] * (v[:, :, c] - grow * torch.matmul(k[:, :, c], S)))
        out[:, :, c] = grow * torch.matmul(q[:, :, c], S) + torch.matmul(P[:, :, c], u)
        left = torch.exp(G[:, :, c, -1:] - G[:, :, c])[..., None]
        S = torch.exp(G[:, :, c, -1])[..., None, None] * S + torch.matmul((left * k[:, :, c]).transpose(-1, -2), u)
    return _delta_done(st, at, there, out.reshape(N, HV, chunks * CHUNK, -1), S)


def _delta_done(st, at, there, out, S):
    o = torch.zeros_like(st["v"])
    o[at[there]] = (st["scale"] * out.transpose(1, 2)[there]).to(o.dtype)
    st["state"][st["slots"].long()] = S
    return {"out": o, "state": st["state"]}


def _recurrent_plain(st):
    at, there, q, k, v, g, b = _delta_inputs(st, st["longest"], torch.float32)
    S = st["state"][st["slots"].long()]
    out = torch.empty_like(v)
    for i in range(st["longest"]):
        S = S * torch.exp(g[:, :, i])[..., None, None]
        u = b[:, :, i, None] * (v[:, :, i] - (k[:, :, i, :, None] * S).sum(-2))
        S = S + k[:, :, i, :, None] * u[:, :, None, :]
        out[:, :, i] = (q[:, :, i, :, None] * S).sum(-2)
    return _delta_done(st, at, there, out, S)


def _adapter_plain(st):
    at, there = _padded(st)
    ids = st["ids"].long()
    safe = ids.clamp(min=0)
    R = st["A"].shape[1]
    live = torch.arange(R, device="cuda")[None, :] < st["ranks"].long()[safe][:, None]
    weight = torch.where(ids >= 0, st["scales"][safe], torch.zeros_like(st["scales"][safe]))[:, None] * live
    x = st["X"].float()[:, at].transpose(0, 1).contiguous()                       # [segments, cols, longest]
    t = torch.matmul(st["A"].float()[safe], x) * weight[..., None]
    d = torch.matmul(st["B"].float()[safe], t)                                    # [segments, rows, longest]
    st["Y"][:, at[there]] += d.transpose(0, 1)[:, there]
    return st["Y"]


def _verify_plain(st):
    drafts, counts = st["drafts"].long(), st["counts"].long()
    B, K = drafts.shape
    V = st["p"].shape[2]
    rows = torch.arange(B, device="cuda")
    p = torch.gather(st["p"][:, :K], 2, drafts[..., None])[..., 0].float()
    q = torch.gather(st["q"], 2, drafts[..., None])[..., 0].float() if st["q"] is not None else torch.ones_like(p)
    asked = torch.arange(K, device="cuda")[None, :] < counts[:, None]
    accepted = torch.cumprod(((st["u"] * q < p) & asked).long(), 1).sum(1)
    x = st["p"][rows, accepted].float()                      # the row that the next token comes from
    refused = accepted < counts
    at = accepted.clamp(max=K - 1)
    if st["q"] is not None:
        less = st["q"][rows, at].float()
    else:
        less = torch.zeros_like(x).scatter_(1, drafts[rows, at][:, None], 1.0)
    left = x - torch.where(refused[:, None], less, torch.zeros_like(less))

    def units(y):
        return (y.clamp(0.0, 1.0) * UNITS).long()
    w = units(left)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, units(x))
    cum = torch.cumsum(w, 1)
    total, m = cum[:, -1], (st["r"] * 2.0 ** 24).long()
    limit = (total >> 24) * m + (((total & 0xffffff) * m) >> 24)                  # floor(total * r), no product past 63 bits
    token = (cum <= limit[:, None]).sum(1)
    token = torch.where(token < V, token, torch.full_like(token, -1))
    place = torch.arange(K + 1, device="cuda")[None, :]
    tokens = torch.nn.functional.pad(drafts, (0, 1))
    tokens = torch.where(place < accepted[:, None], tokens, torch.where(place == accepted[:, None], token[:, None], torch.full_like(tokens, -1)))
    return {"tokens": tokens.to(torch.int32), "accepted": accepted.to(torch.int32)}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"chunked": _chunked_plain, "recurrent": _recurrent_plain, "adapter": _adapter_plain, "verify": _verify_plain}[kind](st)
    from paper_2005_05758_amd import binding as csb
    if kind in ("chunked", "recurrent"):
        call = csb.delta_chunked if kind == "chunked" else csb.delta_recurrent
        out = call(st["q"], st["k"], st["v"], st["g"], st["beta"], scale=st["scale"], starts=st["starts"], state=st["state"],
                   slots=st["slots"])
        return {"out": out, "state": st["state"]}
    if kind == "adapter":
        return csb.adapter_add(st["Y"], st["X"], st["A"], st["B"], st["ids"], starts=st["starts"], scales=st["scales"],
                               ranks=st["ranks"])
    tokens, accepted = csb.verify_drafts(st["p"], st["q"], st["drafts"], st["u"], st["r"], counts=st["counts"])
    return {"tokens": tokens, "accepted": accepted}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("chunked", "recurrent"):
        # S <- a S;  u = beta (v - S^T k);  S <- S + k u^T;  o = scale S^T q, token by token
        at, there, q, k, v, g, b = _delta_inputs(st, st["longest"], torch.float64)
        state = st["state"].double()
        S = state[st["slots"].long()]
        a, out = torch.exp(g), torch.empty_like(v)
        for i in range(st["longest"]):
            S *= a[:, :, i, None, None]
            u = b[:, :, i, None] * (v[:, :, i] - torch.matmul(k[:, :, i, None, :], S)[:, :, 0])
            S.addcmul_(k[:, :, i, :, None], u[:, :, None, :])
            out[:, :, i] = torch.matmul(q[:, :, i, None, :], S)[:, :, 0]
        o = torch.zeros(st["v"].shape, dtype=torch.float64, device="cuda")
        o[at[there]] = st["scale"] * out.transpose(1, 2)[there]
        state[st["slots"].long()] = S
        return {"out": o, "state": state}
    if case["kind"] == "adapter":
        Y, first = st["Y"].double(), st["starts"].tolist()
        for s, a in enumerate(st["ids"].tolist()):
            if a >= 0:
                r, cols = int(st["ranks"][a]), slice(first[s], first[s + 1])
                t = st["A"][a, :r].double() @ st["X"][:, cols].double()
                Y[:, cols] += float(st["scales"][a]) * (st["B"][a, :, :r].double() @ t)
        return Y
    # Whole numbers: request by request on the host.
    K, V = case["drafts"], case["vocab"]
    drafts, counts, u, r = (st[n].cpu().numpy() for n in ("drafts", "counts", "u", "r"))
    tokens, accepted = np.full((case["requests"], K + 1), -1, np.int32), np.zeros(case["requests"], np.int32)
    for b in range(case["requests"]):
        n = 0
        while n < counts[b]:
            d = int(drafts[b, n])
            q = st["q"][b, n, d].float().item() if st["q"] is not None else 1.0
            if not float(np.float32(u[b, n]) * np.float32(q)) < st["p"][b, n, d].float().item():
                break
            tokens[b, n] = d
            n += 1
        row = st["p"][b, n].float().cpu().numpy()
        left = row.copy()
        if n < counts[b] and st["q"] is not None:
            left = row - st["q"][b, n].float().cpu().numpy()
        elif n < counts[b]:
            left[drafts[b, n]] -= np.float32(1.0)
        for weights in (left, row):
            cum = np.cumsum((np.clip(weights, 0.0, 1.0).astype(np.float64) * UNITS).astype(np.int64))
            if cum[-1] > 0:
                limit = int(cum[-1]) * int(float(r[b]) * 2.0 ** 24) >> 24
                tokens[b, n] = np.searchsorted(cum, limit, side="right")
                break
        accepted[b] = n
    return {"tokens": torch.from_numpy(tokens).cuda(), "accepted": torch.from_numpy(accepted).cuda()}


def work(case):
    kind, size = case["kind"], SIZE[case["format"]]
    if kind in ("chunked", "recurrent"):
        N, T, HK, HV, DK, DV = (case[k] for k in ("seqs", "tokens", "heads_k", "heads_v", "dk", "dv"))
        # q, k, v and the output, decay and beta, the states read and written; S^T k, k u^T and S^T q per token
        return {"bytes": T * (2.0 * HK * DK + 2.0 * HV * DV) * size + 8.0 * T * HV + 8.0 * N * HV * DK * DV,
                "flops": 6.0 * T * HV * DK * DV}
    if kind == "adapter":
        rows, cols, n, R = case["rows"], case["cols"], case["batch"], case["rank"]
        # ranks are 3/4 of the largest on average; the result is read and written
        return {"bytes": 0.75 * case["adapters"] * R * (rows + cols) * size + n * (cols * size + rows * 8.0),
                "flops": 2.0 * 0.75 * n * R * (rows + cols)}
    # of all rows only the one that the next token comes from (and its draft's)
    V = case["vocab"]
    return {"bytes": case["requests"] * (V * size * (2.0 if case["draft_probs"] else 1.0) + case["drafts"] * (2.0 * size + 12.0)),
            "flops": case["requests"] * 4.0 * V}
