"""The serving example of selective scans: pruned projections, norms, convolution, scan, sampling and verification as a user's program runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_scan.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serve_scan", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def model(example):
    return example.Model(vocab=60, width=96, layers=2, inner=160, n=8, requests=3)


def states(m):
    return [t.float().clone() for l in m.layers for t in (l.state, l.inputs)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_what_is_tried_is_kept_as_far_as_it_is_accepted(example):
    """A step over drafts leaves the states that the accepted tokens alone leave, to the bfloat16 rounding of the layers' inputs (2^-8, summed in
    another order by products of another batch)."""
    prompts = [[1, 2, 3, 4, 5], [6] * 70, [7, 8]]
    a, b = model(example), model(example)
    starts, tokens = i32([0, 5, 75, 77]), i32(sum(prompts, []))
    pa, pb = a.prompt(tokens, starts), b.prompt(tokens, starts)
    assert torch.equal(pa, pb)
    before = states(a)
    last, drafts = i32([3, 9, 11]), i32([[4, 5, 6], [10, 11, 12], [1, 1, 1]])
    q = torch.full((3, 3, 60), 1.0 / 60, device="cuda")
    u = torch.tensor([[0.0, 0.0, 0.0], [0.0, 1e9, 0.0], [1e9, 0.0, 0.0]], device="cuda")    # all, one, none accepted
    new, accepted = a.step(last, drafts, q, u, torch.full((3,), 0.5, device="cuda"), {"temperature": torch.full((3,), 1.0, device="cuda")})
    assert accepted.tolist() == [3, 1, 0]
    assert new[0, :3].tolist() == [4, 5, 6] and new[1, 0] == 10 and new[1, 2:].tolist() == [-1, -1] and new[2, 1:].tolist() == [-1] * 3
    assert all(0 <= int(new[i, n]) < 60 for i, n in enumerate([3, 1, 0]))
    seqs = [[3, 4, 5, 6], [9, 10], [11]]                 # the same tokens, and no others
    b.run(i32(sum(seqs, [])), True, starts=i32([0, 4, 6, 7]))
    for x, y, z in zip(states(a), states(b), before):
        assert not torch.equal(x, z)
        assert (x - y).abs().max() <= 0.02 * y.abs().max()


def test_prompts_whole_or_token_by_token(example):
    a, b = model(example), model(example)
    t = torch.arange(150, device="cuda", dtype=torch.int32) % 60
    pa = a.run(t, True, starts=i32([0, 1, 140, 150]))[0]
    at = [0, 1, 140, 150]
    for i in range(139):                                 # all requests that still have tokens
        take = [at[s] + i for s in range(3) if at[s] + i < at[s + 1]]
        live = [s for s in range(3) if at[s] + i < at[s + 1]]
        pb = b.run(t[take], True, starts=torch.arange(len(take) + 1, dtype=torch.int32, device="cuda"), slots=i32(live))[0]
        if i == 138:
            assert (pa[139] - pb[0]).abs().max() <= 0.03 * pa.abs().max()
    for x, y in zip(states(a), states(b)):
        assert (x - y).abs().max() <= 0.03 * y.abs().max()


def test_requests_keep_to_themselves(example):
    """Another request's prompt changes nothing of this one's tokens."""
    one = example.serve(model(example), [[1, 2, 3], [4, 5, 6, 7], [8] * 30], 4)[0]
    two = example.serve(model(example), [[1, 2, 3], [40, 50, 6, 7], [8] * 30], 4)[0]
    assert one[0] == two[0] and one[2] == two[2] and all(0 <= x < 60 for row in one for x in row)
    assert all(len(row) >= 5 for row in one)
