"""Products of 8-bit rows of no columns: y is the bias."""

import pytest
import torch

import paper_2406_16282_amd as lmbp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("m", [1, 70])
def test_no_columns_leave_the_bias_alone(m, bad):
    """k = 0: a sum of nothing is 0 whatever the scales are."""
    n = 48
    none = torch.empty(0, dtype=torch.int8, device=DEV)
    scale, w_scale = torch.full((m,), bad, device=DEV), torch.rand(n, device=DEV)
    bias = torch.randn(n, device=DEV)
    for s, ws in ((scale, w_scale), (torch.rand(m, device=DEV), torch.full((n,), bad, device=DEV))):
        y = lmbp.linear_q8_fwd(none.view(m, 0), s, none.view(n, 0), ws, bias, torch.float32)
        assert torch.equal(y, bias.expand(m, n))
        assert (lmbp.linear_q8_fwd(none.view(m, 0), s, none.view(n, 0), ws) == 0).all()
