"""The measured cases of the operators around a recurrent layer of a language model: selective scan and its short
convolution, norms around a block, sampling.

A case is a dict of plain values.  `kind` picks the operator:

  "scan"    selective_scan: the selective state space scan, over whole prompts or a few tokens of many requests
  "conv"    short_conv: the short causal convolution in front of it, its last inputs kept per request
  "norm"    block_norm: a block's output normalised, gated, scaled, added to the residual stream, normalised for the next block
  "sample"  sample: the next token from logits with temperature, top-k, top-p and min-p, from given random numbers

run() computes a case in its plain form, elementary torch operations in 32 bits (the weights of a sample, which are whole
units, in 64); with `own` set it makes the framework's calls.  exact() computes it from the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
CHUNK = 64                   # tokens that the plain form of the scan takes one after the other, all chunks at once
UNITS = 2.0 ** 38            # sampling: weights are counted in whole units of 2^-38 of the largest
EPS = 1e-5


def _scan(name, seqs, tokens, channels, groups, n, fmt, spread):
    """`tokens`: all sequences together.  `spread`: longest over mean length (1: all alike)."""
    return {"name": name, "kind": "scan", "seqs": seqs, "tokens": tokens, "channels": channels, "groups": groups, "n": n,
            "format": fmt, "spread": spread}


def _conv(name, seqs, tokens, channels, width, fmt, spread):
    return {"name": name, "kind": "conv", "seqs": seqs, "tokens": tokens, "channels": channels, "width": width, "format": fmt,
            "spread": spread}


def _norm(name, tokens, width, groups, fmt, form):
    """`form`: "between" (norm of the block's output, residual, norm for the next block; the output comes from a product and the
    result goes into one, both column by column), "heads" (a gated norm of every head), "add" (residual and a norm with the mean)."""
    return {"name": name, "kind": "norm", "tokens": tokens, "width": width, "groups": groups, "format": fmt, "form": form}


def _sample(name, rows, vocab, fmt, filters, probs):
    """`filters`: some of "k", "p", "m" (min-p), in one text.  `probs`: whether the filtered distribution is asked for too."""
    return {"name": name, "kind": "sample", "rows": rows, "vocab": vocab, "format": fmt, "filters": filters, "probs": probs}


def listed():
    return [
        # One long document read at once through a wide layer.
        _scan("scan_long_bf16", 1, 16384, 4096, 1, 16, "bf16", 1.0),
        # The prompts of many requests as a server packs them, of very different lengths.
        _scan("scan_packed_bf16", 48, 16411, 2048, 1, 16, "bf16", 4.0),
        # Full precision, grouped inputs and sizes that fill no tile, as a small research model has them.
        _scan("scan_odd_f32", 5, 1999, 665, 5, 10, "f32", 2.0),
        # Decoding: a full batch of requests, one token each.
        _scan("scan_step_bf16", 64, 64, 4096, 1, 16, "bf16", 1.0),
        # The convolution of those packed prompts.
        _conv("conv_packed_bf16", 48, 16411, 4096, 4, "bf16", 4.0),
        # Requests that bring a few drafted tokens each, an odd batch of them.
        _conv("conv_drafts_f16", 33, 131, 2048, 4, "f16", 2.0),
        # Between two blocks of a prompt's layers, around the large square projection.
        _norm("norm_between_bf16", 2048, 8192, 1, "bf16", "between"),
        # A gated norm of every head behind a recurrence, packed prompts.
        _norm("norm_heads_f16", 16411, 2048, 16, "f16", "heads"),
        # One token: the smallest call, where latency is all there is.
        _norm("norm_one_f32", 1, 4096, 1, "f32", "add"),
        # One request, a vocabulary of odd size, all filters.
        _sample("sample_one_f32", 1, 20011, "f32", "kpm", False),
        # A batch and a large vocabulary, all filters.
        _sample("sample_batch_f32", 64, 131071, "f32", "kpm", False),
        # The distributions that drafts are verified against: a few rows of every request, top-p.
        _sample("sample_probs_bf16", 165, 32003, "bf16", "p", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "scan", "conv", "norm", "norm", "sample", "sample"])
    fmt = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("scan", "conv"):
        if rng.random() < 0.5:                               # prompts
            tokens = _log(rng, 33, 16384)
            seqs = min(_log(rng, 1, 48), max(1, tokens // 8))
        else:                                                # single tokens and drafts
            seqs = _log(rng, 1, 96)
            tokens = seqs if rng.random() < 0.5 else _log(rng, seqs, 6 * seqs)
        spread = round(rng.uniform(1.0, 4.0), 1)
        if kind == "conv":
            c = _conv("", seqs, tokens, _log(rng, 64, 4096), rng.choice([2, 3, 4, 4, 4, 6, 8]), fmt, spread)
        else:
            groups = rng.choice([1, 1, 2, 4])
            most = 4096 * 16 * 16384 // tokens               # no more work than the largest listed
            n = rng.choice([16, 16, 8, 32, _log(rng, 1, 64)])
            channels = min(_log(rng, 64, 4096), max(64, most // n))
            c = _scan("", seqs, tokens, -(-channels // groups) * groups, groups, n, fmt, spread)
    elif kind == "norm":
        form = rng.choice(["between", "between", "heads", "add"])
        width, tokens = _log(rng, 64, 8192), _log(rng, 1, 8192)
        tokens = max(1, min(tokens, 2048 * 8192 // width))
        groups = rng.choice([1, 4, 8, 16]) if form == "heads" else 1
        c = _norm("", tokens, -(-width // groups) * groups, groups, fmt, form)
    else:
        filters = rng.choice(["kpm", "kpm", "k", "p", "m", "kp", ""])
        vocab = _log(rng, 500, 131072)
        rows = max(1, min(_log(rng, 1, 128), 64 * 131071 // vocab))
        c = _sample("", rows, vocab, fmt, filters, rng.random() < 0.4)
    del c["name"]
    return c


def _lengths(seed, n, total, spread):
    """n lengths of `total` together, none of them zero, the longest about spread * mean."""
    g = np.random.Generator(np.random.PCG64(seed))
    w = np.exp(g.uniform(-math.log(spread), 0.0, n)) if spread > 1.0 else np.ones(n)
    cut = np.floor(np.cumsum(w) / w.sum() * (total - n) + 0.5).astype(np.int64)
    return np.diff(np.concatenate([[0], cut])) + 1


def prepare(case, seed):
    t = torch.Generator(device="cuda").manual_seed(seed + 15485863)

    def normal(*shape):
        return torch.randn(shape, generator=t, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=t, device="cuda")

    kind, typ = case["kind"], TYPES[case["format"]]
    if kind in ("scan", "conv"):
        N, T, C = case["seqs"], case["tokens"], case["channels"]
        lengths = _lengths(seed, N, T, case["spread"])
        pool = N + 3                                         # requests sit anywhere in the pool of states
        st = {"case": case, "starts": torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda(),
              "longest": int(lengths.max()), "slots": torch.randperm(pool, generator=t, device="cuda")[:N].to(torch.int32)}
        if kind == "conv":
            W = case["width"]
            return st | {"x": normal(T, C).to(typ), "weight": normal(C, W) * W ** -0.5, "bias": 0.1 * normal(C),
                         "state": normal(pool, W - 1, C).to(typ)}
        G, n = case["groups"], case["n"]
        x = normal(T, C)
        step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(C))       # a channel's usual step, 0.001 to 0.1
        return st | {"x": (x * torch.sigmoid(x)).to(typ), "z": normal(T, C).to(typ), "dt": (0.5 * normal(T, C)).to(typ),
                     "dt_bias": torch.log(torch.expm1(step)), "A": -torch.arange(1, n + 1, device="cuda") * (0.5 + uniform(C, 1)),
                     "B": normal(T, G, n).to(typ), "C": normal(T, G, n).to(typ), "D": 1.0 + 0.1 * normal(C),
                     "state": 0.3 * normal(pool, C, n)}
    if kind == "norm":
        T, W, form = case["tokens"], case["width"], case["form"]
        st = {"case": case, "after_weight": 1.0 + 0.1 * normal(W), "before_weight": 1.0 + 0.1 * normal(W), "before_bias": 0.1 * normal(W)}
        if form == "heads":
            return st | {"y": normal(T, W).to(typ), "gate": normal(T, W).to(typ)}
        if form == "add":
            return st | {"y": normal(T, W).to(typ), "x": 2.0 * normal(T, W).to(typ), "out": torch.empty(T, W, dtype=typ, device="cuda")}
        ld = T + -T % 4                                      # a product's operands: [width, tokens padded to a multiple of 4]
        return st | {"y": normal(W, ld), "x": 2.0 * normal(T, W).to(typ), "scales": 0.1 + uniform(W),
                     "out": torch.empty(T, W, dtype=typ, device="cuda"), "normed": torch.zeros(W, ld, dtype=typ, device="cuda")}
    R, V, f = case["rows"], case["vocab"], case["filters"]

    def some(values, off):                                   # one row in five goes without
        return torch.where(uniform(R) < 0.2, torch.full_like(values, off), values) if R > 1 else values
    return {"case": case, "logits": (3.0 * normal(R, V)).to(typ), "r": uniform(R), "temperature": 0.5 + uniform(R),
            "top_k": some(torch.randint(5, 200, (R,), generator=t, device="cuda"), 0).to(torch.int32) if "k" in f else None,
            "top_p": some(0.7 + 0.29 * uniform(R), 1.0) if "p" in f else None,
            "min_p": some(0.01 + 0.1 * uniform(R), 0.0) if "m" in f else None}


def _of_tokens(st):
    """The sequence of every token and its place in it."""
    first = st["starts"].long()
    seq = torch.repeat_interleave(torch.arange(len(first) - 1, device="cuda"), first.diff(), output_size=st["case"]["tokens"])
    return seq, torch.arange(st["case"]["tokens"], device="cuda") - first[seq]


def _conv_form(st, dtype):
    x, state, W = st["x"].to(dtype), st["state"], st["case"]["width"]
    seq, pos = _of_tokens(st)
    slots, first = st["slots"].long(), st["starts"].long()
    old = state[slots].to(dtype)                             # [sequences, width - 1, channels]
    at = torch.arange(len(x), device="cuda")
    y = st["bias"].to(dtype).expand_as(x).clone()
    for back in range(W):                                    # the input `back` tokens ago
        here = pos >= back
        v = x[torch.where(here, at - back, at)]
        if back:
            v = torch.where(here[:, None], v, old[seq, (W - 1 - back + pos).clamp(max=W - 2)])
        y += st["weight"][:, W - 1 - back].to(dtype) * v
    y = y * torch.sigmoid(y)
    j = torch.arange(W - 1, device="cuda")
    n = first.diff()[:, None]
    src = first[:-1, None] + n - (W - 1) + j                 # the last inputs; those from before the call in `old`
    kept = torch.where((n + j >= W - 1)[..., None], st["x"][src.clamp(0, len(x) - 1)],
                       state[slots[:, None], (j + n).clamp(max=W - 2)])
    new = state.clone()
    new[slots] = kept
    return y, new


def _conv_plain(st):
    y, new = _conv_form(st, torch.float32)
    st["state"].copy_(new)
    return {"out": y.to(st["x"].dtype), "state": st["state"]}


def _scan_plain(st):
    case = st["case"]
    G, n, longest = case["groups"], case["n"], st["longest"]
    L = min(CHUNK, longest)
    chunks = -(-longest // L)
    first, end = st["starts"][:-1, None].long(), st["starts"][1:, None].long()
    at = first + torch.arange(chunks * L, device="cuda")
    there = at < end
    at = torch.where(there, at, torch.zeros_like(at))
    N = len(first)

    def chunked(v, *tail):                                   # [sequences, chunks, L, ...]
        return v[at].float().reshape(N, chunks, L, *tail)
    dt = torch.logaddexp(st["dt"].float() + st["dt_bias"], torch.zeros((), device="cuda"))
    dt = chunked(dt, G, -1) * there.reshape(N, chunks, L, 1, 1)
    x, B, C = chunked(st["x"], G, dt.shape[-1]), chunked(st["B"], G, n), chunked(st["C"], G, n)
    A = st["A"].reshape(G, -1, n)
    h = torch.zeros(N, chunks, *A.shape, device="cuda")
    y = torch.empty_like(x)
    for i in range(L):                                       # from zero, all chunks at once
        h = h * torch.exp(dt[:, :, i, ..., None] * A) + (dt[:, :, i] * x[:, :, i])[..., None] * B[:, :, i, :, None]
        y[:, :, i] = (h * C[:, :, i, :, None]).sum(-1)
    S = st["state"][st["slots"].long()].reshape(N, *A.shape)
    begin = torch.empty_like(h)
    for c in range(chunks):                                  # what each chunk starts from
        begin[:, c] = S
        S = S * torch.exp(dt[:, c].sum(1)[..., None] * A) + h[:, c]
    for i in range(L):                                       # and what is left of it
        begin *= torch.exp(dt[:, :, i, ..., None] * A)
        y[:, :, i] += (begin * C[:, :, i, :, None]).sum(-1)
    out = torch.empty_like(st["x"])
    z = st["z"].float()
    full = torch.empty(z.shape, device="cuda")
    full[at[there]] = y.reshape(N, chunks * L, -1)[there]
    out[:] = (full + st["D"] * st["x"].float()) * (z * torch.sigmoid(z))
    st["state"][st["slots"].long()] = S.reshape(N, -1, n)
    return {"out": out, "state": st["state"]}


def _normed(v, weight, bias, mean):
    if mean:
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * weight
    return v if bias is None else v + bias


def _norm_form(st, dtype):
    """What comes out, not yet rounded: the gated heads, or the residual stream and its norm."""
    form = st["case"]["form"]
    w = st["after_weight"].to(dtype)
    if form == "heads":
        G = st["case"]["groups"]
        y, g = st["y"].to(dtype), st["gate"].to(dtype)
        return _normed(y.unflatten(1, (G, -1)), w.view(G, -1), None, False).flatten(1) * (g * torch.sigmoid(g)), None
    if form == "add":
        r = st["x"].to(dtype) + st["y"].to(dtype)
        return r, _normed(r, st["before_weight"].to(dtype), st["before_bias"].to(dtype), True)
    T = st["case"]["tokens"]
    r = st["x"].to(dtype) + st["scales"].to(dtype) * _normed(st["y"][:, :T].t().to(dtype), w, None, False)
    return r, _normed(r, st["before_weight"].to(dtype), None, False)


def _norm_plain(st):
    form, typ, T = st["case"]["form"], TYPES[st["case"]["format"]], st["case"]["tokens"]
    r, n = _norm_form(st, torch.float32)
    if form == "heads":
        return {"out": r.to(typ)}
    if form == "between":
        st["normed"][:, :T] = n.t().to(typ)
        n = st["normed"]
    st["out"].copy_(r)
    return {"out": st["out"], "normed": n.to(typ)}


def _sample_plain(st):
    s = st["logits"].double()
    R, V = s.shape
    s, order = torch.sort(s, dim=1, descending=True, stable=True)                 # ties: the lowest index first
    w = (torch.exp((s - s[:, :1]) / st["temperature"].double()[:, None]) * UNITS).long()
    place = torch.arange(V, device="cuda")
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        w = torch.where((place < k) | (k <= 0), w, torch.zeros_like(w))
    kept = w > 0
    if st["top_p"] is not None:
        p = st["top_p"][:, None]
        cum = torch.cumsum(w, 1)
        total, m = cum[:, -1:], (p.double() * 2.0 ** 24).long()
        limit = (total >> 24) * m + (((total & 0xffffff) * m) >> 24)              # floor(total * p), no product past 63 bits
        kept &= (cum - w < limit) | (place == 0) | (p >= 1.0)
    if st["min_p"] is not None:
        kept &= w >= (st["min_p"].double() * UNITS).long()[:, None]
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, torch.zeros_like(w)))     # by index again
    cum = torch.cumsum(w, 1)
    total, m = cum[:, -1], (st["r"].double() * 2.0 ** 24).long()
    limit = (total >> 24) * m + (((total & 0xffffff) * m) >> 24)
    token = (cum <= limit[:, None]).sum(1).to(torch.int32)
    if not st["case"]["probs"]:
        return {"tokens": token}
    return {"tokens": token, "probs": (w.double() / total[:, None].double()).to(st["logits"].dtype)}


def run(st):
    kind, case = st["case"]["kind"], st["case"]
    if not own:
        return {"scan": _scan_plain, "conv": _conv_plain, "norm": _norm_plain, "sample": _sample_plain}[kind](st)
    from paper_2005_05758_amd import binding as csb
    if kind == "scan":
        out = csb.selective_scan(st["x"], st["dt"], st["A"], st["B"], st["C"], D=st["D"], z=st["z"], dt_bias=st["dt_bias"],
                                 starts=st["starts"], state=st["state"], slots=st["slots"])
        return {"out": out, "state": st["state"]}
    if kind == "conv":
        out = csb.short_conv(st["x"], st["weight"], st["bias"], starts=st["starts"], state=st["state"], slots=st["slots"])
        return {"out": out, "state": st["state"]}
    if kind == "norm":
        if case["form"] == "heads":
            out, _ = csb.block_norm(st["y"], gate=st["gate"], after="rms", after_weight=st["after_weight"], groups=case["groups"], eps=EPS)
            return {"out": out}
        if case["form"] == "add":
            r, n = csb.block_norm(st["y"], x=st["x"], before="mean", before_weight=st["before_weight"], before_bias=st["before_bias"],
                                  eps=EPS, out=st["out"])
            return {"out": r, "normed": n}
        T = case["tokens"]
        r, _ = csb.block_norm(st["y"][:, :T].t(), x=st["x"], after="rms", after_weight=st["after_weight"], scales=st["scales"], before="rms",
                              before_weight=st["before_weight"], eps=EPS, out=st["out"], normed=st["normed"][:, :T].t())
        return {"out": r, "normed": st["normed"]}
    got = csb.sample(st["logits"], st["r"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"],
                     probs=case["probs"])
    return {"tokens": got[0], "probs": got[1]} if case["probs"] else {"tokens": got}


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "conv":
        # token by token would be the same sums; the padded sequence of each request, convolved
        W, first = case["width"], st["starts"].tolist()
        out, state = torch.empty(st["x"].shape, dtype=torch.float64, device="cuda"), st["state"].double()
        for i, s in enumerate(st["slots"].tolist()):
            v = torch.cat([state[s], st["x"][first[i]:first[i + 1]].double()])
            y = st["bias"].double() + sum(v[j:j + first[i + 1] - first[i]] * st["weight"][:, j].double() for j in range(W))
            out[first[i]:first[i + 1]] = y / (1.0 + torch.exp(-y))
            state[s] = v[len(v) - (W - 1):]
        return {"out": out, "state": state}
    if kind == "scan":
        # h <- exp(dt A) h + dt x B;  y = C h + D x, gated, token by token, all sequences at once
        G, n = case["groups"], case["n"]
        first, lengths = st["starts"][:-1].long(), st["starts"].long().diff()
        A = st["A"].double().reshape(G, -1, n)
        state = st["state"].double()
        S = state[st["slots"].long()].reshape(-1, *A.shape)
        out = torch.empty(st["x"].shape, dtype=torch.float64, device="cuda")
        order = torch.argsort(lengths, descending=True)      # the sequences that still have tokens come first
        S, first = S[order], first[order]
        live = sorted(lengths.tolist(), reverse=True)
        m = len(live)
        bias, D = st["dt_bias"].double(), st["D"].double()
        for i in range(st["longest"]):
            while live[m - 1] <= i:
                m -= 1
            at = first[:m] + i
            dt = st["dt"][at].double() + bias
            dt = (torch.clamp(dt, min=0.0) + torch.log1p(torch.exp(-dt.abs()))).reshape(m, G, -1, 1)
            x, z = st["x"][at].double(), st["z"][at].double()
            S[:m] *= torch.exp(dt * A)
            S[:m] += dt * x.reshape(m, G, -1, 1) * st["B"][at].double()[:, :, None]
            y = (S[:m] * st["C"][at].double()[:, :, None]).sum(-1).reshape(m, -1) + D * x
            out[at] = y * z / (1.0 + torch.exp(-z))
        state[st["slots"].long()[order]] = S.reshape(len(order), -1, n)
        return {"out": out, "state": state}
    if kind == "norm":
        r, n = _norm_exact(st, case)
        return {"out": r} if n is None else {"out": r, "normed": n}
    # Whole numbers: row by row on the host.
    tokens, probs = [], []
    asked = {k: st[k].tolist() if st[k] is not None else None for k in ("top_k", "top_p", "min_p", "temperature", "r")}
    rows = st["logits"].double().cpu().numpy()
    for i, s in enumerate(rows):
        order = np.lexsort((np.arange(len(s)), -s))
        w = (np.exp((s - s.max()) / asked["temperature"][i]) * UNITS).astype(np.int64)
        keep = order
        if asked["top_k"] is not None and asked["top_k"][i] > 0:
            keep = keep[:asked["top_k"][i]]
        if asked["top_p"] is not None and asked["top_p"][i] < 1.0:
            before = np.cumsum(w[keep]) - w[keep]
            limit = int(w[keep].sum()) * int(asked["top_p"][i] * 2 ** 24) >> 24
            keep = keep[:max(1, int(np.searchsorted(before, limit, side="left")))]
        if asked["min_p"] is not None:
            keep = keep[w[keep] >= int(asked["min_p"][i] * UNITS)]
        left = np.zeros_like(w)
        left[keep] = w[keep]
        cum = np.cumsum(left)
        limit = int(cum[-1]) * int(asked["r"][i] * 2 ** 24) >> 24
        tokens.append(int(np.searchsorted(cum, limit, side="right")))
        if case["probs"]:
            probs.append(left / cum[-1])
    got = {"tokens": torch.tensor(tokens, dtype=torch.int32, device="cuda")}
    return got | {"probs": torch.from_numpy(np.stack(probs)).cuda()} if case["probs"] else got


def _norm_exact(st, case):
    d = {k: v.double() for k, v in st.items() if isinstance(v, torch.Tensor)}
    T, W = case["tokens"], case["width"]

    def unit(v):                                             # rows of length sqrt(size)
        return v / torch.sqrt(v.square().sum(-1, keepdim=True) / v.shape[-1] + EPS)
    if case["form"] == "heads":
        y = unit(d["y"].reshape(T * case["groups"], -1)).reshape(T, W) * d["after_weight"]
        return y * d["gate"] / (1.0 + torch.exp(-d["gate"])), None
    if case["form"] == "add":
        r = d["x"] + d["y"]
        c = r - r.sum(-1, keepdim=True) / W
        return r, unit(c) * d["before_weight"] + d["before_bias"]
    r = d["x"] + unit(d["y"].t()[:T].contiguous()) * d["after_weight"] * d["scales"]
    n = torch.zeros(d["y"].shape, dtype=torch.float64, device="cuda")
    n[:, :T] = (unit(r) * d["before_weight"]).t()
    return r, n


def work(case):
    kind, size = case["kind"], SIZE[case["format"]]
    if kind == "conv":
        N, T, C, W = (case[k] for k in ("seqs", "tokens", "channels", "width"))
        return {"bytes": 2.0 * T * C * size + 2.0 * N * (W - 1) * C * size + 4.0 * C * (W + 1), "flops": T * C * (2.0 * W + 4)}
    if kind == "scan":
        N, T, C, G, n = (case[k] for k in ("seqs", "tokens", "channels", "groups", "n"))
        # x, step, gate and output, B and C; the states read and written.  Per state and token: two products, an exponential, two sums of products
        return {"bytes": T * (4.0 * C + 2.0 * G * n) * size + 8.0 * N * C * n + 4.0 * C * (n + 2), "flops": 7.0 * T * C * n + 12.0 * T * C}
    if kind == "norm":
        T, W, form = case["tokens"], case["width"], case["form"]
        if form == "heads":
            return {"bytes": 3.0 * T * W * size, "flops": 8.0 * T * W}
        first = 4.0 if form == "between" else size           # the block's output; a product's is binary32
        return {"bytes": T * W * (first + 3.0 * size), "flops": 9.0 * T * W}
    R, V = case["rows"], case["vocab"]
    return {"bytes": R * V * size * (2.0 if case["probs"] else 1.0) + 20.0 * R, "flops": 4.0 * R * V}
