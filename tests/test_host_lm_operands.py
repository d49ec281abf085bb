"""The language-model operators' checks of where their operands are, with stand-ins for tensors of several devices.  No GPU."""
import pytest
import torch

from paper_2005_05758_amd import binding


class Stand:
    def __init__(self, device, grad=False):
        self.device_number, self.is_cuda, self.requires_grad = device, device >= 0, grad

    def get_device(self):
        return self.device_number


@pytest.fixture(autouse=True)
def device_one(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)


def test_all_operands_lie_on_the_current_device():
    a, b = Stand(1), Stand(1)
    assert binding._operands((a, None, b), None, a) == 1
    for floats, others in (((Stand(0), a), ()), ((a, Stand(0)), ()), ((a,), (Stand(0),)), ((a, b), (None, Stand(-1)))):
        with pytest.raises(AssertionError, match="current device"):
            binding._operands(floats, *others)
    with pytest.raises(AssertionError):
        binding._operands((Stand(-1), a))


def test_an_operand_that_requires_a_gradient():
    with pytest.raises(AssertionError, match="gradient"):
        binding._operands((Stand(1), None, Stand(1, grad=True)))
    with torch.no_grad():
        assert binding._operands((Stand(1), Stand(1, grad=True))) == 1
