"""Where relu is flat its gradient is zero, whatever the gradient behind it holds."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [64, 61])
@pytest.mark.parametrize("r", [0, 8, 48])
def test_infinities_and_nan_behind_a_dead_unit_add_nothing(r, n, dtype):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(n + r)
    z, dy = torch.randn(100, n, generator=gen).to(dtype).cuda(), torch.randn(100, n, generator=gen).to(dtype).cuda()
    z[3] = 0.0
    t = torch.randn(100, r, generator=gen).to(dtype).cuda() if r else None
    want = L.loract_linear_backward(torch.where(z > 0, dy, torch.zeros_like(dy)), z, act="relu", lora_t=t)
    dead = z <= 0
    dy[dead] = torch.tensor([float("inf"), -float("inf"), float("nan")], dtype=dtype, device="cuda")[torch.arange(int(dead.sum()), device="cuda") % 3]
    got = L.loract_linear_backward(dy, z, act="relu", lora_t=t)
    assert torch.isfinite(got[0]).all() and all(a is b or torch.equal(a, b) for a, b in zip(got, want))
