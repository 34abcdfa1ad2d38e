"""Adapters of many requests, both routes (in the order the tokens come, and ordered by adapter first): the digits of X A."""
import pytest
import torch

import paper_2509_23472_amd as L
from test_gpu_lora_requests import BF, F32, _ids

pytestmark = pytest.mark.gpu
# (tokens, rank, adapters): few tokens of a small rank in the order they come; more of them, a larger rank, or much of A and B ordered
ROUTES = [(1, 16, 3), (20, 8, 3), (64, 32, 4), (300, 16, 5), (50, 64, 4), (1000, 33, 7)]


@pytest.mark.parametrize("m,r,count", ROUTES)
def test_float32_results_keep_24_digits_of_xa(m, r, count):
    """X A of numbers whose products and partial sums are whole multiples of 2^-16 below 2^8: 24 digits, so that every order of the sum is exact; each
    column of B has a single power of two.  Y is s X A moved by it, without any rounding."""
    gen = torch.Generator(device="cuda").manual_seed(m + r)
    digits = torch.randint(0, 128, (m, 3), generator=gen, device="cuda") * 2 + 1                  # odd, 8 bits: all 24 digits of X A are used
    sign = torch.randint(0, 2, (m, 1), generator=gen, device="cuda") * 2 - 1
    x = torch.zeros(m, 40, device="cuda")
    x[:, [3, 17, 39]] = digits.float() * sign * torch.tensor([2.0 ** 0, 2.0 ** -8, 2.0 ** -16], device="cuda")
    a = torch.exp2(torch.arange(r, device="cuda") % 5.0).repeat(count, 40, 1)                       # column k: 2^(k mod 5)
    n_out = 200
    hot = torch.randint(0, r, (count, n_out), generator=gen, device="cuda")
    b = torch.zeros(count, r, n_out, device="cuda").scatter_(1, hot[:, None], 0.25)
    ids = _ids("mixed", m, count, gen)
    got = L.loract_lora_requests(x.to(BF), a.to(BF), b.to(BF), ids, torch.full((count,), 2.0, device="cuda"), out_dtype=F32)
    t = x.double().sum(1)
    want = 0.5 * t[:, None] * torch.exp2(hot % 5.0).double()[ids.clamp(min=0).long()]
    want[ids < 0] = 0
    assert torch.equal(got.double(), want), (got.double() - want).abs().max()
