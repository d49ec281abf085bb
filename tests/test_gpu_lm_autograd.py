"""The language-model operators beside autograd, which they take no part in: what would lose a gradient is refused, what they change in place is
known to have changed."""
import sys

import pytest
import torch

from paper_2005_05758_amd import adapter_add, delta_chunked, delta_recurrent, verify_drafts

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def delta_operands():
    unit = lambda: torch.nn.functional.normalize(torch.randn(20, 1, 16, device="cuda"), dim=-1)   # noqa: E731
    return [unit(), unit(), torch.randn(20, 2, 8, device="cuda"), -torch.rand(20, 2, device="cuda"), torch.rand(20, 2, device="cuda")]


def adapter_operands():
    return [torch.randn(24, 8, device="cuda"), torch.randn(32, 8, device="cuda"), torch.randn(1, 4, 32, device="cuda"), torch.randn(1, 24, 4, device="cuda")]


def verify_operands():
    p = torch.softmax(torch.randn(2, 4, 50, device="cuda"), -1)
    return [p, p[:, :3].contiguous(), i32([[1, 2, 3], [4, 5, 6]]), torch.rand(2, 3, device="cuda"), torch.rand(2, device="cuda")]


CALLS = {
    "chunked": (delta_operands, range(5), lambda ops: delta_chunked(*ops)),
    "recurrent": (delta_operands, range(5), lambda ops: delta_recurrent(*ops)),
    "adapter": (adapter_operands, range(4), lambda ops: adapter_add(*ops, i32([0]), starts=i32([0, 8]))),
    "verify": (verify_operands, (0, 1), lambda ops: verify_drafts(*ops)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_operands_that_require_a_gradient(name):
    """Refused where gradients are enabled, taken where they are not."""
    say(f"[autograd] {name}")
    make, places, call = CALLS[name]
    for i in places:
        ops = make()
        ops[i].requires_grad_(True)
        with pytest.raises(AssertionError, match="gradient"):
            call(ops)
        with torch.no_grad():
            got = call(ops)
        assert not any(t.requires_grad for t in (got if isinstance(got, tuple) else (got,)) if t is not ops[0])
    with torch.inference_mode():
        call(make())
    call(make())
    torch.cuda.synchronize()


def test_what_is_changed_in_place_is_known_to_have_changed():
    say("[autograd] in place")
    w = torch.ones(24, 8, device="cuda", requires_grad=True)
    Y, X, A, B = adapter_operands()
    loss = (w * Y).sum()                                 # keeps Y for w's gradient
    adapter_add(Y, X, A, B, i32([0]), starts=i32([0, 8]))
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    for form in (delta_chunked, delta_recurrent):
        ops = delta_operands()
        for what in ("state", "state_out", "out"):
            t = torch.zeros(20, 2, 8, device="cuda") if what == "out" else torch.zeros(1, 2, 16, 8, device="cuda")
            w = torch.ones_like(t, requires_grad=True)
            loss = (w * t).sum()
            form(*ops, **{what: t})
            with pytest.raises(RuntimeError, match="inplace"):
                loss.backward()
        state = torch.zeros(1, 2, 16, 8, device="cuda")
        w = torch.ones_like(state, requires_grad=True)
        loss = (w * state).sum()
        form(*ops, state=state, state_out=None)          # read only
        loss.backward()
    torch.cuda.synchronize()


def test_operands_on_the_host():
    say("[autograd] host operands")
    ops = delta_operands()
    for kw in (dict(starts=i32([0, 20], "cpu")), dict(lens=i32([20], "cpu")), dict(slots=i32([0], "cpu")), dict(state=torch.zeros(1, 2, 16, 8))):
        with pytest.raises(AssertionError):
            delta_chunked(*ops, **kw)
    Y, X, A, B = adapter_operands()
    for a, ids in ((A.cpu(), i32([0])), (A, i32([0], "cpu"))):
        with pytest.raises(AssertionError):
            adapter_add(Y, X, a, B, ids, starts=i32([0, 8]))
    p, q, d, u, r = verify_operands()
    for bad in ((p.cpu(), q, d, u, r), (p, q.cpu(), d, u, r), (p, q, d.cpu(), u, r), (p, q, d, u, r.cpu())):
        with pytest.raises(AssertionError):
            verify_drafts(*bad)
    torch.cuda.synchronize()
