"""Keys of no heads: what the forward pass accepts has a backward pass, with a gradient of zero for the gain."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gain", [False, True])
def test_keys_of_no_heads(gain):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(1)
    q, dq = torch.randn(5, 2, 64, generator=gen).cuda(), torch.randn(5, 2, 64, generator=gen).cuda()
    none, table = torch.zeros(5, 0, 64, device="cuda"), L.loract_rope_table(5, 64)
    gamma = torch.ones(64, device="cuda") if gain else None
    y, k = L.loract_qknorm_rope_forward(q, none, gamma, gamma, table)
    assert k.shape == none.shape and torch.equal(y, L.loract_qknorm_rope_forward(q, None, gamma, None, table)[0])
    got = L.loract_qknorm_rope_backward(q, none, gamma, gamma, table, dq, none)
    want = L.loract_qknorm_rope_backward(q, None, gamma, None, table, dq, None)
    assert torch.equal(got[0], want[0]) and got[1].shape == none.shape
    assert (got[2] is None and got[3] is None) if not gain else torch.equal(got[2], want[2]) and not got[3].any()
