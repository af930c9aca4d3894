"""What the module of a norm and its 8-bit layers refuses: layers whose own call would not run
(the module reads their weights and calls the operators itself). Nothing here reaches a GPU."""

import pytest
import torch

from paper_2406_16282_amd.nn import LinearQ8, MSRMSNormLinearQ8


def layer():
    return LinearQ8(torch.zeros(4, 6, dtype=torch.int8), torch.ones(4))


class Adapted(LinearQ8):
    def forward(self, x):
        return super().forward(x) + x.sum()


class Wrapper(torch.nn.Module):
    """A wrapper that hands out the attributes of the layer inside."""

    def __init__(self, inner):
        super().__init__()
        self.inner = inner
        self.weight, self.scale, self.bias = inner.weight, inner.scale, inner.bias

    def forward(self, x):
        return self.inner(x)


def test_layers_with_a_call_of_their_own():
    with pytest.raises(TypeError, match="LinearQ8"):
        MSRMSNormLinearQ8([layer(), Adapted(torch.zeros(4, 6, dtype=torch.int8), torch.ones(4))])
    with pytest.raises(TypeError, match="LinearQ8"):
        MSRMSNormLinearQ8([Wrapper(layer())])


@pytest.mark.parametrize("change", ["wrapped", "adapted", "forward"])
def test_layers_that_are_replaced_later(change):
    block, x = MSRMSNormLinearQ8([layer(), layer()]), torch.zeros(2, 6)
    if change == "wrapped":
        block.layers[1] = Wrapper(block.layers[1])
    elif change == "adapted":
        block.layers[1].__class__ = Adapted
    else:
        block.layers[1].forward = lambda x: x
    with pytest.raises(TypeError, match="LinearQ8"):
        block(x)


@pytest.mark.parametrize("register", ["register_forward_hook", "register_forward_pre_hook",
                                      "register_full_backward_hook", "register_full_backward_pre_hook"])
def test_hooks_that_would_not_run(register):
    block, x = MSRMSNormLinearQ8([layer(), layer()]), torch.zeros(2, 6)
    handle = getattr(block.layers[0], register)(lambda *a: None)
    with pytest.raises(RuntimeError, match="hook"):
        block(x)
    handle.remove()
    with pytest.raises(ValueError, match="GPU tensor"):   # the call itself again
        block(x)


def test_hooks_of_the_module_itself_run():
    block, seen = MSRMSNormLinearQ8([layer()]), []
    block.register_forward_pre_hook(lambda m, a: seen.append(a))
    with pytest.raises(ValueError, match="GPU tensor"):
        block(torch.zeros(2, 6))
    assert len(seen) == 1
