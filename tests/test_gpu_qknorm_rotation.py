"""The backward rotation of float32 gradients where its two terms nearly cancel."""
import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [128, 64, 30])
def test_differences_of_nearly_equal_terms(d, interleaved):
    """Inputs of zeros: dx = Rot^T dy / sqrt(eps).  Relative, whatever cancels: the rotation two roundings of 2^-24 (of the sum, and with what
    the first product's rounding left), the reciprocal root three, the product one, and two to spare."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(d)
    m, heads, eps = 256, 24, 2.0 ** -20
    dy = torch.randn(m, heads, d, generator=gen)
    table = L.loract_rope_table(m, d)
    x = torch.zeros(m, heads, d, device="cuda")
    dx = L.loract_qknorm_rope_backward(x, None, None, None, table, dy.cuda(), None, eps=eps, interleaved=interleaved)[0]
    want = ref.rotate(dy.double(), table.double().cpu(), interleaved, back=True) / eps ** 0.5
    ref.check(dx, want, 8 * 2.0 ** -24 * want.abs(), "dx")
