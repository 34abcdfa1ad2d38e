"""What loract_adamw takes for eps: the quotient's reciprocal is the hardware's, to which a number below 2^-126 is zero."""
import pytest
import torch

import paper_2509_23472_amd as L
from test_adamw_abi import INVALID, _call

LEAST = 2.0 ** -126


@pytest.mark.parametrize("eps", [1e-40, 1e-45, 1e-300, LEAST * (1 - 2.0 ** -24)])
def test_an_eps_that_would_count_as_zero_is_refused(eps):
    assert _call(eps=eps) == INVALID


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype", [torch.float32, torch.bfloat16])
def test_the_smallest_eps_keeps_what_has_no_gradient(p_dtype, bits):
    p = torch.randn(700, device="cuda").to(p_dtype)
    params, before = [p], p.clone()
    L.loract_adamw(params, [torch.zeros(700, device="cuda")], L.loract_adamw_state(params, bits=bits), step=1, lr=1e-3, eps=LEAST, weight_decay=0.0)
    assert torch.equal(p, before)
