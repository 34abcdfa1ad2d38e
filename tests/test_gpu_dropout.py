"""loract_dropout: the mask of its definition, on every alignment, and nothing but the mask."""
import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu


def _check(m, n, p, seed, dtype, residual, pad=0, shift=0):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(seed & 0xFFFF)
    x = torch.randn(m, n, generator=gen).to(dtype)
    res = torch.randn(m, n, generator=gen).to(dtype) if residual else None
    place = lambda t: torch.empty((m, n + pad + shift), dtype=dtype, device="cuda")[:, shift:shift + n].copy_(t)
    y = L.loract_dropout(place(x), p, seed, residual=None if res is None else place(res), out=place(torch.zeros(m, n)))
    fac = ref.drop_factors(m, n, p, seed & (2 ** 64 - 1))
    want = x.double() * fac + (res.double() if residual else 0.0)
    ref.check(y, want, 2.0 ** -22 * (x.double().abs() * fac + want.abs()) + 1.01 * ref.U[dtype] * want.abs(), "Y")
    if not residual:
        assert torch.equal(y.cpu() == 0, (fac == 0) | (x == 0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9999])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 3), (2, 5), (7, 64), (33, 96), (5, 1030), (197, 768), (300, 7)])
def test_mask(m, n, p, residual, dtype):
    _check(m, n, p, 12345, dtype, residual)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,shift", [(8, 8), (4, 4), (3, 1), (1, 0)])
def test_strides(pad, shift, dtype):
    _check(37, 96, 0.3, 2 ** 64 - 5, dtype, True, pad, shift)
    _check(37, 97, 0.3, -7, dtype, False, pad, shift)


def test_gradient_is_the_same_call():
    """D is linear: <C, D(X + h V)> differs by h <D(C), V>; with h = 1 and factors of 2 every step but the sums is exact."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(1)
    x, v, c = (torch.randint(-8, 9, (64, 52), generator=gen).float().cuda() for _ in range(3))
    d = lambda t: L.loract_dropout(t, 0.5, 99)
    num = (c * (d(x + v) - d(x))).double().sum()
    assert num == (d(c) * v).double().sum() and num != 0


def test_dropped_values_are_zero_whatever_they_were_and_in_place():
    import paper_2509_23472_amd as L
    keep = ref.drop_factors(40, 64, 0.5, 3) > 0
    for bad in (float("nan"), float("inf"), -3e38):
        y = L.loract_dropout(torch.full((40, 64), bad, device="cuda"), 0.5, 3).cpu()
        assert (y[~keep] == 0).all() and not (y[keep] == 0).any()
    x = torch.randn(40, 64, device="cuda")
    want = L.loract_dropout(x, 0.5, 3)
    got = L.loract_dropout(x, 0.5, 3, out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)


def test_no_elements_and_other_seeds():
    import paper_2509_23472_amd as L
    assert L.loract_dropout(torch.zeros((0, 8), device="cuda"), 0.1, 0).shape == (0, 8)
    x = torch.ones(256, 1024, device="cuda")
    a, b = L.loract_dropout(x, 0.25, 1) > 0, L.loract_dropout(x, 0.25, 2) > 0
    # kept fractions 0.75 and, of both, 0.75^2: six deviations of a binomial over 2^18 elements
    for kept, want in ((a, 0.75), (b, 0.75), (a & b, 0.5625)):
        assert abs(kept.double().mean().item() - want) < 6 * (want * (1 - want) / 2 ** 18) ** 0.5


def test_offsets_past_32_bits():
    import paper_2509_23472_amd as L
    m, n = 66000, 33000
    x = torch.ones((m, n), dtype=torch.bfloat16, device="cuda")
    L.loract_dropout(x, 0.5, 8, out=x)
    rows = [0, 65075, 65076, m - 1]
    assert torch.equal(x[rows].double().cpu(), ref.drop_factors(m, n, 0.5, 8, rows))
