"""Serving a small recurrent language model: pruned projections, an adapter per request, the gated delta rule, drafted tokens.

Random weights and prompts.  A layer's projections are pruned matrices with bfloat16 values applied by csb_spmm_bfloat, the layer
input's one with the adapters of the requests on top; its recurrence is the gated delta rule, chunk by chunk over the prompts
and token by token behind them.  A step tries the last token and a few drafts of every request at once: the recurrence runs over them without
keeping the states, the target's probabilities verify the drafts, and the states are then taken as far as the drafts were accepted.

    python examples/serve_delta.py            on an MI355X, after building the library
"""
import os
import sys
import time

import numpy as np
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2005_05758_amd import VAL_BF16, CsbMatrix, adapter_add, delta_chunked, delta_recurrent, verify_drafts  # noqa: E402


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


def columns(x):
    """[tokens, width] as the products take it: [width, tokens] bfloat16, the tokens padded to a multiple of 4."""
    return F.pad(x.t(), (0, -x.shape[0] % 4)).bfloat16().contiguous()


class Layer:
    def __init__(self, rng, width, heads_k, heads_v, dk, dv, requests, adapters, rank):
        self.hk, self.hv, self.dk, self.dv = heads_k, heads_v, dk, dv
        self.sizes = [heads_k * dk, heads_k * dk, heads_v * dv, heads_v, heads_v]       # q, k, v, decay, beta
        self.into, self.back = pruned(rng, sum(self.sizes), width), pruned(rng, width, heads_v * dv)
        t = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
        self.A = (torch.randn(adapters, rank, width, generator=t, device="cuda") * width ** -0.5).bfloat16()
        self.B = (torch.randn(adapters, sum(self.sizes), rank, generator=t, device="cuda") * 0.1).bfloat16()
        self.state = torch.zeros(requests, heads_v, dk, dv, device="cuda")

    def project(self, x, ids, starts):
        """What the recurrence takes of tokens x [tokens, width] (request s: starts[s] .. starts[s + 1] - 1, adapter ids[s])."""
        X = columns(F.layer_norm(x, x.shape[1:]))
        Y = self.into.spmm_bfloat(X)
        adapter_add(Y, X, self.A, self.B, ids, starts=starts)
        q, k, v, g, beta = Y[:, :len(x)].t().contiguous().split(self.sizes, dim=1)
        q, k = (F.normalize(F.silu(y.unflatten(1, (self.hk, self.dk))), dim=-1).bfloat16() for y in (q, k))
        return q, k, v.unflatten(1, (self.hv, self.dv)).bfloat16(), -0.1 * F.softplus(g), torch.sigmoid(beta)

    def output(self, x, o):
        return x + self.back.spmm_bfloat(columns(F.layer_norm(o.flatten(1).float(), (self.hv * self.dv,))))[:, :len(x)].t()


class Model:
    """`requests` states per layer; a request keeps its adapter (-1: none) as long as it lives."""

    def __init__(self, seed=0, vocab=500, width=512, layers=2, heads_k=4, heads_v=8, dk=64, dv=64, requests=16, adapters=4, rank=16):
        rng = np.random.default_rng(seed)
        self.layers = [Layer(rng, width, heads_k, heads_v, dk, dv, requests, adapters, rank) for _ in range(layers)]
        t = torch.Generator(device="cuda").manual_seed(seed)
        self.embed, self.head = (torch.randn(vocab, width, generator=t, device="cuda") for _ in range(2))
        self.bigram = self.probabilities(self.embed)           # the draft's probabilities of the next token: what the model says without its layers
        self.ids = torch.tensor([i % (adapters + 1) - 1 for i in range(requests)], dtype=torch.int32, device="cuda")

    def probabilities(self, x):
        return torch.softmax(F.layer_norm(x, x.shape[1:]) @ self.head.t() * (2.0 * self.head.shape[1] ** -0.5), -1)

    def run(self, tokens, starts, call, keep):
        """Probabilities behind every token; `keep`: whether the states are.  Also what each layer's recurrence took."""
        x, taken = self.embed[tokens.long()], []
        for l in self.layers:
            ins = l.project(x, self.ids, starts)
            taken.append(ins)
            o = call(*ins, starts=starts, state=l.state, **({} if keep else {"state_out": None}))
            x = l.output(x, o)
        return self.probabilities(x), taken

    def prompt(self, tokens, starts):
        """Takes whole prompts in; returns the probabilities of each request's next token."""
        p, _ = self.run(tokens, starts, delta_chunked, True)
        return p[starts[1:].long() - 1]

    def step(self, last, drafts, draft_probs, u, r):
        """Tries last [requests] and drafts [requests, n] behind it, keeps what is accepted.  Returns (tokens [requests, n + 1]: the accepted
        drafts, one more token, -1; accepted [requests])."""
        N, n = drafts.shape
        tokens = torch.cat([last[:, None], drafts], 1).flatten()
        starts = torch.arange(N + 1, dtype=torch.int32, device="cuda") * (n + 1)
        p, taken = self.run(tokens, starts, delta_recurrent, False)
        new, accepted = verify_drafts(p.view(N, n + 1, -1), draft_probs, drafts, u, r)
        for l, ins in zip(self.layers, taken):                 # the last token and the accepted drafts
            delta_recurrent(*ins, starts=starts, lens=accepted + 1, state=l.state)
        return new, accepted


def serve(model, prompts, steps, drafts=3, seed=0):
    """Prompts (lists of tokens) in, `steps` steps of every request; returns the tokens of each and the share of drafts accepted."""
    t = torch.Generator(device="cuda").manual_seed(seed)
    N = len(prompts)
    starts = torch.tensor(np.cumsum([0] + [len(p) for p in prompts]), dtype=torch.int32, device="cuda")
    p = model.prompt(torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda"), starts)
    none = torch.zeros(N, 0, dtype=torch.int32, device="cuda")
    last = verify_drafts(p[:, None], None, none, none.float(), torch.rand(N, generator=t, device="cuda"))[0][:, 0]    # no drafts: a sample
    said, taken = [last[:, None]], 0
    for _ in range(steps):
        d, q, at = [], [], last
        for _ in range(drafts):
            q.append(model.bigram[at.long()])
            at = torch.multinomial(q[-1], 1, generator=t)[:, 0].int()
            d.append(at)
        new, accepted = model.step(last, torch.stack(d, 1), torch.stack(q, 1), torch.rand(N, drafts, generator=t, device="cuda"),
                                   torch.rand(N, generator=t, device="cuda"))
        said.append(new)
        taken = taken + accepted.sum()
        last = torch.gather(new, 1, accepted[:, None].long())[:, 0]
    rows = torch.cat(said, 1).tolist()
    return [[x for x in row if x >= 0] for row in rows], float(taken) / max(1, steps * drafts * N)


if __name__ == "__main__":
    model = Model()
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, 500, int(n)).tolist() for n in rng.integers(5, 400, 16)]
    serve(model, prompts, 2)                                   # first launches
    torch.cuda.synchronize()
    t = time.perf_counter()
    said, share = serve(model, prompts, 20)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"{len(prompts)} requests, {sum(map(len, prompts))} prompt tokens, {sum(map(len, said))} tokens said in {t * 1e3:.1f} ms; "
          f"{100 * share:.0f} % of the drafts accepted; the first request: {said[0][:12]}")
