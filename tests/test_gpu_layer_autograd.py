"""The operators around a recurrent layer beside autograd, which they take no part in: what would lose a gradient is refused, what they change in
place is known to have changed; operands on the host are refused."""
import sys

import pytest
import torch

from paper_2005_05758_amd import block_norm, sample, selective_scan, short_conv

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def rnd(*s):
    return torch.randn(*s, device="cuda")


CALLS = {
    "conv": (lambda: [rnd(9, 16), rnd(16, 4), rnd(16), torch.zeros(1, 3, 16, device="cuda")],
             lambda x, w, b, s: short_conv(x, w, b, state=s)),
    "scan": (lambda: [rnd(9, 16), rnd(9, 16), -rnd(16, 8).abs(), rnd(9, 1, 8), rnd(9, 1, 8), rnd(16), rnd(9, 16), rnd(16), torch.zeros(1, 16, 8, device="cuda")],
             lambda x, dt, A, B, C, D, z, b, s: selective_scan(x, dt, A, B, C, D=D, z=z, dt_bias=b, state=s)),
    "norm": (lambda: [rnd(9, 16), rnd(9, 16), rnd(9, 16), rnd(16), rnd(16), rnd(16), rnd(16), rnd(16)],
             lambda y, g, x, a, b, c, d, e: block_norm(y, gate=g, x=x, after="rms", after_weight=a, after_bias=b, scales=c, before="rms", before_weight=d, before_bias=e)),
    "sample": (lambda: [rnd(3, 50), torch.rand(3, device="cuda"), torch.ones(3, device="cuda"), torch.ones(3, device="cuda"), torch.zeros(3, device="cuda")],
               lambda l, r, t, p, q: sample(l, r, temperature=t, top_p=p, min_p=q, probs=True)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_operands_that_require_a_gradient(name):
    """Refused where gradients are enabled, taken where they are not."""
    say(f"[autograd] {name}")
    make, call = CALLS[name]
    for i in range(len(make())):
        ops = make()
        ops[i].requires_grad_(True)
        with pytest.raises(AssertionError, match="gradient"):
            call(*ops)
        with torch.no_grad():
            got = call(*ops)
        assert not any(t.requires_grad for t in (got if isinstance(got, tuple) else (got,)))
    with torch.inference_mode():
        call(*make())
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", sorted(CALLS))
def test_operands_on_the_host(name):
    say(f"[autograd] {name} on the host")
    make, call = CALLS[name]
    for i in range(len(make())):
        ops = make()
        ops[i] = ops[i].cpu()
        with pytest.raises(AssertionError):
            call(*ops)
    x, w, b, s = CALLS["conv"][0]()
    for kw in (dict(starts=i32([0, 9], "cpu")), dict(lens=i32([9], "cpu")), dict(slots=i32([0], "cpu"))):
        with pytest.raises(AssertionError):
            short_conv(x, w, b, **kw)
    with pytest.raises(AssertionError):
        sample(rnd(3, 50), torch.rand(3, device="cuda"), top_k=i32([1, 2, 3], "cpu"))
    torch.cuda.synchronize()


def changed(call, t):
    """Whether autograd learns that `call` changes t."""
    w = torch.ones_like(t, requires_grad=True)
    loss = (w * t).sum()                                 # keeps t for w's gradient
    call(t)
    try:
        loss.backward()
        return False
    except RuntimeError as e:
        assert "inplace" in str(e)
        return True


def test_what_is_changed_in_place_is_known_to_have_changed():
    say("[autograd] in place")
    x, w, b, s = CALLS["conv"][0]()
    x2, dt, A, B, C, D, z, bias, state = CALLS["scan"][0]()
    assert changed(lambda t: short_conv(x, w, b, state=t), s.clone()) and changed(lambda t: short_conv(x, w, b, state=s, state_out=t), s.clone())
    assert changed(lambda t: short_conv(x, w, b, out=t), rnd(9, 16)) and not changed(lambda t: short_conv(x, w, b, state=t, state_out=None), s.clone())
    scan = lambda **kw: selective_scan(x2, dt, A, B, C, **kw)            # noqa: E731
    assert changed(lambda t: scan(state=t), state.clone()) and changed(lambda t: scan(state=state, state_out=t), state.clone())
    assert changed(lambda t: scan(out=t), rnd(9, 16)) and not changed(lambda t: scan(state=t, state_out=None), state.clone())
    assert changed(lambda t: block_norm(x, out=t), rnd(9, 16)) and changed(lambda t: block_norm(x=x, before="rms", normed=t), rnd(9, 16))
    assert changed(lambda t: block_norm(x, x=t, out=t), rnd(9, 16)) and not changed(lambda t: block_norm(x, x=t), rnd(9, 16))
    assert changed(lambda t: sample(t, probs=t), rnd(3, 50)) and not changed(lambda t: sample(t, probs=True), rnd(3, 50))
    torch.cuda.synchronize()
