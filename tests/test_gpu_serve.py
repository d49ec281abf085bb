"""The serving example: pruned projections, adapters, the delta rule and verification as a user's program runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_delta.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("serve_delta", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def model(example):
    return example.Model(vocab=60, width=96, layers=2, heads_k=1, heads_v=2, dk=32, dv=48, requests=3, adapters=2, rank=4)


def states(m):
    return [l.state.clone() for l in m.layers]


def test_what_is_tried_is_kept_as_far_as_it_is_accepted(example):
    """A step over drafts leaves the states that the accepted tokens alone leave, to the bfloat16 rounding of the layers' inputs (2^-8, summed in
    another order by products of another batch)."""
    prompts = [[1, 2, 3, 4, 5], [6] * 70, [7, 8]]
    a, b = model(example), model(example)
    starts = torch.tensor([0, 5, 75, 77], dtype=torch.int32, device="cuda")
    tokens = torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda")
    pa, pb = a.prompt(tokens, starts), b.prompt(tokens, starts)
    assert torch.equal(pa, pb)
    before = states(a)
    last = torch.tensor([3, 9, 11], dtype=torch.int32, device="cuda")
    drafts = torch.tensor([[4, 5, 6], [10, 11, 12], [1, 1, 1]], dtype=torch.int32, device="cuda")
    q = torch.full((3, 3, 60), 1.0 / 60, device="cuda")
    u = torch.tensor([[0.0, 0.0, 0.0], [0.0, 1e9, 0.0], [1e9, 0.0, 0.0]], device="cuda")    # all, one, none accepted
    new, accepted = a.step(last, drafts, q, u, torch.full((3,), 0.5, device="cuda"))
    assert accepted.tolist() == [3, 1, 0]
    assert new[0, :3].tolist() == [4, 5, 6] and new[1, 0] == 10 and new[1, 2:].tolist() == [-1, -1] and new[2, 1:].tolist() == [-1] * 3
    assert all(0 <= int(new[i, n]) < 60 for i, n in enumerate([3, 1, 0]))
    # the same tokens, and no others
    seqs = [[3, 4, 5, 6], [9, 10], [11]]
    starts = torch.tensor([0, 4, 6, 7], dtype=torch.int32, device="cuda")
    b.run(torch.tensor(sum(seqs, []), dtype=torch.int32, device="cuda"), starts, example.delta_recurrent, True)
    for x, y, z in zip(states(a), states(b), before):
        assert not torch.equal(x, z)
        assert (x - y).abs().max() <= 0.02 * y.abs().max()
    torch.cuda.synchronize()


def test_prompts_chunk_by_chunk_or_token_by_token(example):
    a, b = model(example), model(example)
    t = torch.arange(150, device="cuda", dtype=torch.int32) % 60
    starts = torch.tensor([0, 1, 140, 150], dtype=torch.int32, device="cuda")
    pa, _ = a.run(t, starts, example.delta_chunked, True)
    pb, _ = b.run(t, starts, example.delta_recurrent, True)
    for x, y in zip(states(a), states(b)):
        assert (x - y).abs().max() <= 0.02 * y.abs().max()
    assert (pa - pb).abs().max() <= 0.02


def test_requests_keep_to_themselves(example):
    """Another request's prompt changes nothing of this one's tokens."""
    one = example.serve(model(example), [[1, 2, 3], [4, 5, 6, 7], [8] * 30], 4)[0]
    two = example.serve(model(example), [[1, 2, 3], [40, 50, 6, 7], [8] * 30], 4)[0]
    assert one[0] == two[0] and one[2] == two[2] and all(0 <= x < 60 for row in one for x in row)
    assert all(len(row) >= 5 for row in one)
