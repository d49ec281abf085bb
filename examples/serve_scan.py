"""Serving a small language model of selective scans: pruned projections, norms between them, drafted tokens, sampling.

Random weights and prompts.  Projections are pruned matrices with bfloat16 values applied by csb_spmm_bfloat, which takes and leaves its operands
column by column; block_norm turns them over as it normalises: a layer's output is added to the residual stream and normalised for the next layer in one call.  A layer
is a projection, the short convolution, a second projection that makes the scan's steps and its B and C, the selective scan, a gated norm and the projection
back.  A step tries the last token and a few drafts of every request at once, without keeping the states; sample gives the
distributions of drafts and target, verify_drafts compares them, and the states are then taken as far as the drafts were accepted.

    python examples/serve_scan.py            on an MI355X, after building the library
"""
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2005_05758_amd import VAL_BF16, CsbMatrix, block_norm, sample, selective_scan, short_conv, verify_drafts  # noqa: E402


def pruned(rng, rows, cols, block=32, keep=0.35):
    """A projection whose blocks keep some of their rows and columns, as the matrix cores read it."""
    grid = (-(-rows // block), -(-cols // block))
    mask = np.kron(np.ones(grid), np.ones((block, block)))[:rows, :cols]
    for i in range(grid[0]):
        for j in range(grid[1]):
            part = mask[i * block:(i + 1) * block, j * block:(j + 1) * block]
            part *= (rng.random((part.shape[0], 1)) < keep ** 0.5) * (rng.random((1, part.shape[1])) < keep ** 0.5)
    m = CsbMatrix((rng.normal(0, (cols * keep) ** -0.5, (rows, cols)) * mask).astype(np.float32), block, block)
    m.set_value_format(VAL_BF16)
    m.plan()
    return m.upload()


def columns(width, tokens):
    """A product's operand [width, tokens padded to a multiple of 4], and its tokens as rows."""
    X = torch.zeros(width, tokens + -tokens % 4, dtype=torch.bfloat16, device="cuda")
    return X, X[:, :tokens].t()


def rows(Y, tokens, first, end):
    """Rows `first` to `end` of a product's result, token by token in bfloat16."""
    out = torch.empty(tokens, end - first, dtype=torch.bfloat16, device="cuda")
    return block_norm(Y[first:end, :tokens].t(), out=out)[0]


class Layer:
    def __init__(self, rng, width, inner, n, conv, requests):
        self.inner, self.n = inner, n
        self.into, self.mid, self.back = pruned(rng, 2 * inner, width), pruned(rng, inner + 2 * n, inner), pruned(rng, width, inner)
        t = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
        rnd = lambda *s: torch.randn(*s, generator=t, device="cuda")   # noqa: E731
        self.weight, self.bias = rnd(inner, conv) * conv ** -0.5, 0.1 * rnd(inner)
        self.A = -torch.arange(1, n + 1, device="cuda").float().repeat(inner, 1)
        self.D, self.gain, self.before = torch.ones(inner, device="cuda"), 1 + 0.1 * rnd(inner), 1 + 0.1 * rnd(width)
        self.dt_bias = torch.log(torch.expm1(torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(inner, generator=t, device="cuda"))))
        self.inputs = torch.zeros(requests, conv - 1, inner, dtype=torch.bfloat16, device="cuda")
        self.state = torch.zeros(requests, inner, n, device="cuda")

    def recur(self, x, z, tokens, keep, **seq):
        """The layer behind its first projection; `keep`: whether the states are."""
        kept = {} if keep else {"state_out": None}
        xc = short_conv(x, self.weight, self.bias, state=self.inputs, **seq, **kept)
        X, view = columns(self.inner, tokens)
        block_norm(xc, out=view)
        p = rows(self.mid.spmm_bfloat(X), tokens, 0, self.inner + 2 * self.n)
        dt, B, C = p.split([self.inner, self.n, self.n], dim=1)
        o = selective_scan(xc, dt, self.A, B.unflatten(1, (1, self.n)), C.unflatten(1, (1, self.n)), D=self.D, dt_bias=self.dt_bias,
                           state=self.state, **seq, **kept)
        X, view = columns(self.inner, tokens)
        block_norm(o, gate=z, after="rms", after_weight=self.gain, out=view)
        return self.back.spmm_bfloat(X)


class Model:
    def __init__(self, seed=0, vocab=500, width=512, layers=2, inner=1024, n=16, conv=4, requests=16):
        rng = np.random.default_rng(seed)
        self.layers = [Layer(rng, width, inner, n, conv, requests) for _ in range(layers)]
        t = torch.Generator(device="cuda").manual_seed(seed)
        self.embed, self.head = (torch.randn(vocab, width, generator=t, device="cuda") for _ in range(2))
        self.last = torch.ones(width, device="cuda")
        self.bigram = self.embed @ self.head.t() * (2.0 * width ** -0.5 / math.sqrt(2.0))     # what the drafts are made from

    def run(self, tokens, keep, **seq):
        """Logits behind every token, and what each layer's recurrence took."""
        T, taken = len(tokens), []
        h = self.embed[tokens.long()].clone()
        X, view = columns(h.shape[1], T)
        block_norm(x=h, before="rms", before_weight=self.layers[0].before, normed=view)
        for l, nxt in zip(self.layers, self.layers[1:] + [None]):
            Y = l.into.spmm_bfloat(X)
            x, z = rows(Y, T, 0, l.inner), rows(Y, T, l.inner, 2 * l.inner)
            taken.append((x, z))
            Y = l.recur(x, z, T, keep, **seq)
            if nxt is not None:                              # the residual stream, in place, and the next layer's operand
                X, view = columns(h.shape[1], T)
                block_norm(Y[:, :T].t(), x=h, scale=0.5, before="rms", before_weight=nxt.before, out=h, normed=view)
            else:
                _, n = block_norm(Y[:, :T].t(), x=h, scale=0.5, before="rms", before_weight=self.last, out=h)
        return n @ self.head.t() * (2.0 * h.shape[1] ** -0.5), taken

    def prompt(self, tokens, starts):
        """Takes whole prompts in; returns the logits of each request's next token."""
        logits, _ = self.run(tokens, True, starts=starts)
        return logits[starts[1:].long() - 1]

    def step(self, last, drafts, draft_probs, u, r, filters):
        """Tries last [requests] and drafts [requests, n] behind it, keeps what is accepted.  Returns (tokens [requests, n + 1]: the accepted
        drafts, one more token, -1; accepted [requests])."""
        N, n = drafts.shape
        tokens = torch.cat([last[:, None], drafts], 1).flatten()
        starts = torch.arange(N + 1, dtype=torch.int32, device="cuda") * (n + 1)
        logits, taken = self.run(tokens, False, starts=starts)
        p = sample(logits, probs=True, **{k: v.repeat_interleave(n + 1) for k, v in filters.items()})
        new, accepted = verify_drafts(p.view(N, n + 1, -1), draft_probs, drafts, u, r)
        for l, (x, z) in zip(self.layers, taken):            # the last token and the accepted drafts
            l.recur(x, z, len(tokens), True, starts=starts, lens=accepted + 1)
        return new, accepted


def serve(model, prompts, steps, drafts=3, seed=0):
    """Prompts (lists of tokens) in, `steps` steps of every request; returns the tokens of each and the share of drafts accepted."""
    t = torch.Generator(device="cuda").manual_seed(seed)
    N = len(prompts)
    filters = {"temperature": torch.full((N,), 0.8, device="cuda"), "top_k": torch.full((N,), 40, dtype=torch.int32, device="cuda"),
               "top_p": torch.full((N,), 0.95, device="cuda")}
    starts = torch.tensor(np.cumsum([0] + [len(p) for p in prompts]), dtype=torch.int32, device="cuda")
    logits = model.prompt(torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda"), starts)
    last = sample(logits, torch.rand(N, generator=t, device="cuda"), **filters)
    said, taken = [last[:, None]], 0
    for _ in range(steps):
        d, q, at = [], [], last
        for _ in range(drafts):
            at, probs = sample(model.bigram[at.long()], torch.rand(N, generator=t, device="cuda"), probs=True, **filters)
            d.append(at)
            q.append(probs)
        new, accepted = model.step(last, torch.stack(d, 1), torch.stack(q, 1), torch.rand(N, drafts, generator=t, device="cuda"),
                                   torch.rand(N, generator=t, device="cuda"), filters)
        said.append(new)
        taken = taken + accepted.sum()
        last = torch.gather(new, 1, accepted[:, None].long())[:, 0]
    lines = torch.cat(said, 1).tolist()
    return [[x for x in line if x >= 0] for line in lines], float(taken) / max(1, steps * drafts * N)


if __name__ == "__main__":
    model = Model()
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, 500, int(n)).tolist() for n in rng.integers(5, 400, 16)]
    serve(model, prompts, 2)                                 # first launches
    torch.cuda.synchronize()
    t = time.perf_counter()
    said, share = serve(model, prompts, 20)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"{len(prompts)} requests, {sum(map(len, prompts))} prompt tokens, {sum(map(len, said))} tokens said in {t * 1e3:.1f} ms; "
          f"{100 * share:.0f} % of the drafts accepted; the first request: {said[0][:12]}")
