"""Verification of drafted tokens (csb_verify_drafts): whole numbers, so every result equals the definition's."""
import math
import sys

import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_2005_05758_amd import verify_drafts
from paper_2005_05758_amd.binding import lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def inputs(seed, N, K, V, fmt, spread=2.0, apart=0.7):
    t = torch.Generator().manual_seed(seed)
    logits = spread * torch.randn(N, K + 1, V, generator=t)
    p = torch.softmax(logits, -1).to(TYPES[fmt])
    q = torch.softmax(logits[:, :K] + apart * torch.randn(N, K, V, generator=t), -1).to(TYPES[fmt])
    drafts = torch.multinomial(q.float().reshape(-1, V) + 1e-20, 1, generator=t).view(N, K).int() if K else torch.zeros(N, 0, dtype=torch.int32)
    return p, q, drafts, torch.rand(N, K, generator=t), torch.rand(N, generator=t)


def check(p, q, drafts, u, r, counts=None, place=lambda x: x.cuda()):
    N, K1, V = p.shape
    say(f"[verify] {p.dtype} {N} requests, {K1 - 1} drafts, vocabulary {V}, counts={counts}")
    tokens, accepted = verify_drafts(place(p), place(q) if q is not None else None, drafts.cuda(), u.cuda(), r.cuda(),
                                     counts=torch.tensor(counts, dtype=torch.int32, device="cuda") if counts is not None else None)
    torch.cuda.synchronize()
    wt, wa = ref.verify(p.float().numpy(), q.float().numpy() if q is not None else None, drafts.numpy(), u.numpy(), r.numpy(),
                        counts if counts is not None else [K1 - 1] * N)
    assert np.array_equal(accepted.cpu().numpy(), wa)
    assert np.array_equal(tokens.cpu().numpy(), wt)
    return wt, wa


@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("N,K,V", [(1, 1, 1), (1, 1, 2), (3, 0, 17), (5, 4, 255), (2, 3, 256), (4, 7, 1023), (33, 2, 1025), (3, 70, 40), (6, 5, 20011), (2, 1, 131071)])
def test_shapes(fmt, N, K, V):
    p, q, d, u, r = inputs(N + K + V, N, K, V, fmt)
    check(p, q, d, u, r)
    check(p, None, d, u, r)
    g = np.random.default_rng(V)
    check(p, q, d, u, r, counts=[int(x) for x in g.integers(-1, K + 2, N)])


def test_the_draws_follow_the_target():
    """Many requests of one and the same pair of rows: the tokens that come first are distributed as the target's
    (chi-square over 8 tokens, 20000 draws: below 40 with a probability of 1 - 2e-6)."""
    N, V = 20000, 8
    p, q, _, u, r = inputs(3, 1, 1, V, "f32", spread=1.0, apart=1.0)
    t = torch.Generator().manual_seed(8)
    d = torch.multinomial(q[0, 0], N, replacement=True, generator=t).int().view(N, 1)
    tokens, _ = verify_drafts(p.expand(N, 2, V).contiguous().cuda(), q.expand(N, 1, V).contiguous().cuda(), d.cuda(),
                              torch.rand(N, 1, generator=t).cuda(), torch.rand(N, generator=t).cuda())
    seen = np.bincount(tokens[:, 0].cpu().numpy(), minlength=V)
    want = p[0, 0].double().numpy() * N
    assert ((seen - want) ** 2 / want).sum() < 40


def test_rows_at_their_edges():
    """No weight left, no weight at all, all on one token, ties between a number and a boundary, numbers of 0 and 1."""
    V = 600
    p, q = torch.zeros(9, 2, V), torch.zeros(9, 1, V)
    p[0, 0, 5] = 0.5                                     # p = q, and the draft is refused (u = 1 is not below p / q)
    q[0, 0, 5] = 0.5
    # request 1: nothing anywhere: -1
    p[2, 0, V - 1] = 1.0                                 # all on the last token, r just below 1
    p[3, 0, 0] = 1.0
    p[4, 0, :4] = 0.25                                   # r on a boundary of the sums: the next token
    p[5, 0, :] = math.nan                                # NaN counts nothing
    p[5, 0, 77] = 0.5
    p[6, 0, 3], p[6, 0, 9] = math.inf, 0.25              # a weight counts 1 at most
    p[7, 0, 2], p[7, 0, 4] = -0.5, 2.0 ** -38            # negative ones count nothing; one unit is enough
    p[8, 0, 2], q[8, 0, 2] = 1.0, 0.0                    # a draft that its model gave nothing: accepted where p has any
    p[:, 1, 1] = 1.0
    d = torch.tensor([5, 7, 9, 9, 9, 9, 9, 9, 2], dtype=torch.int32).view(9, 1)
    u = torch.full((9, 1), 1.0)
    r = torch.tensor([0.3, 0.3, 1 - 2.0 ** -24, 0.0, 0.5, 0.9, 0.5, 0.9, 0.9])
    wt, wa = check(p, q, d, u, r)
    assert wt[:, 0].tolist() == [5, -1, V - 1, 0, 2, 77, 9, 4, 2] and wa.tolist() == [0] * 6 + [1, 0, 1]   # (draft 9 of request 6: q is 0)
    check(p, q, d, u, torch.tensor([1.0, 2.0, -1.0, math.nan, math.inf, 1.0, 0.0, 1.0, 0.0]).nan_to_num(0.0, 1.0))
    wt, wa = check(p, None, d, u, r)
    assert wt[:, 0].tolist() == [5, -1, V - 1, 0, 2, 77, 3, 4, 2] and wa.tolist() == [0] * 9


@pytest.mark.parametrize("V", [24575, 24576, 24577, 40000])
def test_rows_at_their_edges_in_large_vocabularies(V):
    """The same where one workgroup's share of a row ends and where several take it."""
    p, q, d, u, r = inputs(V, 6, 1, V, "f32")
    p[0, 0], u[0] = q[0, 0], 1.0                         # p = q and the draft is refused: p's own weights
    p[1, 0] = q[1, 0] = 0.0                              # nothing anywhere
    p[2, 0] = 0.0
    p[2, 0, V - 1], u[2], r[2] = 1.0, 1.0, 1 - 2.0 ** -24
    p[3, 0, 1:] = math.nan
    u[3], r[3] = 1.0, 0.0
    p[4, 0] = p[4, 1] = 0.0
    p[4, 0, d[4, 0]] = p[4, 1, 16384] = 1.0              # accepted, the next token one of a kind
    q[5, 0], u[5] = 1.0, 1.0                             # q above p everywhere
    check(p, q, d, u, r)
    check(p, None, d, u, r)


def test_drafts_outside_the_vocabulary():
    p, q, d, u, r = inputs(4, 4, 3, 100, "f32")
    d[0, 0], d[1, 1], d[2, 2] = -1, 100, 2 ** 31 - 1
    check(p, q, d, u, r)
    check(p, None, d, u, r)


def test_largest_and_smallest_numbers():
    """Every weight of a row at its most, in a vocabulary of 2^20: sums of 2^58 units."""
    V = 1 << 20
    p = torch.ones(2, 1, V)
    r = torch.tensor([0.75, 1 - 2.0 ** -24])
    wt, _ = check(p, None, torch.zeros(2, 0, dtype=torch.int32), torch.zeros(2, 0), r)
    assert wt[:, 0].tolist() == [786432, V - 1]


@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_strides_and_alignment(fmt):
    p, q, d, u, r = inputs(5, 4, 3, 1030, fmt)

    def wide(x):
        y = torch.full((x.shape[0], x.shape[1], 1037), math.nan, dtype=x.dtype, device="cuda")
        y[:, :, :1030] = x.cuda()
        return y[:, :, :1030]

    def shifted(x):
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        y.copy_(x)
        return y
    check(p, q, d, u, r, place=wide)
    check(p, q, d, u, r, place=shifted)


def test_stream_and_graph():
    p, q, d, u, r = (x.cuda() for x in inputs(6, 8, 4, 5000, "f32"))

    def once(stream=None):
        torch.cuda.synchronize()
        got = verify_drafts(p, q, d, u, r, stream=stream)
        torch.cuda.synchronize()
        return got
    want = once()
    got = once(torch.cuda.Stream())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = verify_drafts(p, q, d, u, r)
    for _ in range(3):
        u.copy_(torch.rand_like(u))
        r.copy_(torch.rand_like(r))
        want = once()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])


def test_rows_past_32_bits():
    """More than 2^31 probabilities: the last request's rows are found."""
    N, V = 17, 1 << 24
    p = torch.zeros(N, 8, V, device="cuda")
    p[N - 1, :, V - 1] = 1.0
    d = torch.full((N, 7), V - 1, dtype=torch.int32, device="cuda")
    tokens, accepted = verify_drafts(p, None, d, torch.full((N, 7), 0.5, device="cuda"), torch.full((N,), 0.5, device="cuda"))
    torch.cuda.synchronize()
    assert accepted.tolist() == [0] * (N - 1) + [7] and tokens[-1].tolist() == [V - 1] * 8 and tokens[0].tolist() == [-1] * 8


def test_refusals():
    p, q, d, u, r = (x.cuda() for x in inputs(7, 2, 3, 64, "f32"))
    out, ws = torch.empty(64, dtype=torch.int32, device="cuda"), torch.empty(4096, dtype=torch.uint8, device="cuda")
    names = "type p ldp q ldq draft u r count n_req n_draft vocab tokens accepted ws stream".split()
    good = dict(zip(names, [0, p.data_ptr(), 64, q.data_ptr(), 64, d.data_ptr(), u.data_ptr(), r.data_ptr(), None, 2, 3, 64, out.data_ptr(),
                            out.data_ptr() + 128, ws.data_ptr(), None]))

    def call(**change):
        return lib().csb_verify_drafts(*({**good, **change}[n] for n in names))
    assert lib().csb_verify_workspace_bytes(2, 64) <= ws.numel()
    assert call() == 0 and call(n_req=0) == 0 and call(q=None) == 0
    for change in (dict(type=9), dict(p=None), dict(draft=None), dict(u=None), dict(r=None), dict(tokens=None), dict(accepted=None), dict(ws=None),
                   dict(ldp=63), dict(ldq=63), dict(n_req=-1), dict(n_draft=-1), dict(vocab=0), dict(ws=ws.data_ptr() + 8), dict(p=p.data_ptr() + 2)):
        assert call(**change) == -1, change
    assert call(vocab=(1 << 24) + 1, ldp=1 << 25, ldq=1 << 25) == -4
    assert lib().csb_verify_workspace_bytes(0, 64) == 0 and lib().csb_verify_workspace_bytes(2, 0) == 0
    with pytest.raises(AssertionError):
        verify_drafts(p, q[:, :2], d, u, r)
    with pytest.raises(AssertionError):
        verify_drafts(p, q.half(), d, u, r)
    torch.cuda.synchronize()


def test_refusals_of_sizes():
    p, q, d, u, r = (x.cuda() for x in inputs(9, 2, 3, 64, "f32"))
    out, ws = torch.empty(64, dtype=torch.int32, device="cuda"), torch.empty(4096, dtype=torch.uint8, device="cuda")
    for n_req, vocab in (((1 << 21) + 1, 64), (1 << 20, 1 << 24)):
        assert lib().csb_verify_drafts(0, p.data_ptr(), vocab, q.data_ptr(), vocab, d.data_ptr(), u.data_ptr(), r.data_ptr(), None, n_req, 3, vocab,
                                       out.data_ptr(), out.data_ptr() + 128, ws.data_ptr(), None) == -4
    torch.cuda.synchronize()
