"""Linear maps with more outputs than one direction of a launch has room for."""
import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_in,layout", [(5, "nt"), (9, "nt"), (9, "nn")])
def test_more_than_65535_columns_of_tiles(n_in, layout, dtype):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(n_in)
    m, n_out = 35, 64 * 65535 + 129 + 2                    # (n_out no multiple of a piece: the general tiles)
    x = torch.randn(m, n_in, generator=gen).to(dtype)
    w = torch.randn(n_out, n_in, generator=gen).to(dtype)
    y = L.loract_linear(x.cuda(), (w if layout == "nt" else w.t().contiguous()).cuda(), act="relu", w_transposed=layout == "nn")
    at = torch.cat([torch.arange(0, 200), torch.arange(64 * 65535 - 100, n_out), torch.randint(0, n_out, (20000,), generator=gen)])
    want, pre, perr = ref.linear(x.double(), w[at].double(), act_name="relu")
    ref.check(y[:, at.cuda()], want, ref.linear_bound(want, pre, perr, dtype), "Y")


@pytest.mark.parametrize("n_out", [(1 << 27) - 16, 1 << 27])
def test_one_token_and_very_many_outputs(n_out):
    """Both sides of what the thin kernels' launch has room for."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(1, 8, generator=gen).bfloat16(), torch.randn(1 << 20, 8, generator=gen).bfloat16()
    big = torch.empty((n_out, 8), dtype=torch.bfloat16, device="cuda")
    for i in range(0, n_out, 1 << 20):
        part = big[i:i + (1 << 20)]
        part.copy_(w[:len(part)])
    y = L.loract_linear(x.cuda(), big)
    want, pre, perr = ref.linear(x.double(), w.double())
    bound = ref.linear_bound(want, pre, perr, torch.bfloat16)
    for i in (0, n_out // (1 << 20) // 2, (n_out - 1) // (1 << 20)):
        part = y[:, i << 20:(i + 1) << 20]
        ref.check(part, want[:, :part.shape[1]], bound[:, :part.shape[1]], "Y")


def test_backward_of_the_longest_row():
    import paper_2509_23472_amd as L
    n = 1 << 30
    dy = torch.empty((1, n), device="cuda")
    for i in range(64):
        dy[:, i << 24:(i + 1) << 24] = torch.arange(1 << 24, device="cuda") + i
    dp, db, _ = L.loract_linear_backward(dy)
    assert torch.equal(dp, dy) and torch.equal(db, dy[0])
