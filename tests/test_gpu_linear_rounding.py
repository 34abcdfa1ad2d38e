"""How far the sums of float32 products stray."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n_in,n_out", [(3001, 1030, 770), (1000, 1024, 500), (300, 200, 1000)])
def test_small_tiles_round_in_two_chains(m, n_in, n_out):
    """A chain that adds K products of variance v rounds partial sums of size sqrt(i v), each by 2^-24 / sqrt(6) of itself (uniform over a last
    place, which is between one and two such units): an rms of 0.29 K 2^-24 sqrt(v), 0.29 sqrt(K) of the result's.  Two chains of K / 2:
    0.205 sqrt(K).  The bound lies between them."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(n_in)
    x, w = torch.randn(m, n_in, generator=gen), torch.randn(n_out, n_in, generator=gen)
    want = (x.double() @ w.double().t())
    y = L.loract_linear(x.cuda(), w.cuda()).double().cpu()
    assert ((y - want).square().mean() / want.square().mean()).sqrt() < 0.245 * n_in ** 0.5 * 2.0 ** -24
