"""Adapters of many requests, both routes (in the order the tokens come, and ordered by adapter first): the digits of X A, infinite elements
of B, tokens whose adapter is not in the pool, what is not finite."""
import pytest
import torch

import paper_2509_23472_amd as L
from test_gpu_lora_requests import BF, F32, INF, NAN, _check, _ids, _make

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


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("m,r,count", ROUTES)
def test_infinite_elements_of_b(m, r, count, dtype, out_dtype):
    """t inf = +-inf by the sign of t, whatever t's digits: numbers of bf16 (X of one element that is not zero, A of powers of two), and any others."""
    x, a, b, scales, res, gen = _make(m, 130, 72, r, count, dtype, m + 1, out_dtype)
    x[::2] = 0
    x[::2, 5] = torch.randn(len(x[::2]), generator=gen, device="cuda").to(dtype)
    a[:, 5] = torch.exp2(torch.randint(-3, 4, (count, r), generator=gen, device="cuda").float()).to(dtype)
    scales.fill_(0.5)
    b[:, r // 2, 7], b[:, 0, 30], b[:, r - 1, 71] = INF, -INF, INF
    ids = _ids("mixed", m, count, gen)
    ids[0] = 0
    got = L.loract_lora_requests(x, a, b, ids, scales, residual=res, out_dtype=out_dtype)
    live, far = ids >= 0, torch.tensor([7, 30, 71], device="cuda")
    near = torch.ones(72, dtype=torch.bool, device="cuda")
    near[far] = False
    _check(got[:, near], x, a, b[:, :, near], ids, scales, res[:, near])
    # b's other elements of these columns are finite: the signs are those of X A at the infinite one, which is no zero and far from it
    for j, k, sign in ((7, r // 2, 1), (30, 0, -1), (71, r - 1, 1)):
        t = (x.double() * a[ids.clamp(min=0).long(), :, k].double()).sum(1) * sign
        sure = live & (t.abs() > 1e-6)
        assert sure.sum() >= live.sum() - 1 and torch.equal(got[sure, j].double(), t[sure].sign() * INF), j
    assert torch.equal(got[~live], res[~live])
    x[:] = 0                                                     # 0 inf is no number
    got = L.loract_lora_requests(x, a, b, ids, scales, residual=res, out_dtype=out_dtype)
    assert torch.isnan(got[live][:, far]).all() and torch.equal(got[live][:, near], res[live][:, near]) and torch.equal(got[~live], res[~live])


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("how", ["residual", "in place", "no residual"])
@pytest.mark.parametrize("m,r,count", ROUTES[1:])
def test_ids_past_the_pool(m, r, count, how, dtype, out_dtype):
    x, a, b, scales, res, gen = _make(m, 64, 200, r, count, dtype, 6, out_dtype)
    ids = _ids("mixed", m, count, gen)
    past = torch.tensor([4, 11, m // 2, m - 1], device="cuda")
    ids[past] = torch.tensor([count, 2 ** 31 - 1, 77, count], dtype=torch.int32, device="cuda")
    ids[[0, m - 2]] = -1
    if how == "in place":
        got = L.loract_lora_requests(x, a, b, ids, scales, residual=(out := res.clone()), out=out, out_dtype=out_dtype)
        assert got is out
    else:
        got = L.loract_lora_requests(x, a, b, ids, scales, residual=res if how == "residual" else None, out_dtype=out_dtype)
    assert torch.isnan(got[past]).all()
    assert torch.equal(got[ids < 0], res[ids < 0] if how != "no residual" else torch.zeros_like(res[ids < 0]))
    _check(got, x, a, b, ids, scales, res if how != "no residual" else None)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,r", [(300, 16), (50, 64), (777, 33)])
def test_what_is_not_finite_stays_with_its_own_where_tokens_are_ordered(m, r, dtype):
    """Several tokens of every adapter share its tile with the token that holds NaN."""
    x, a, b, scales, res, gen = _make(m, 200, 136, r, 8, dtype, 7)
    ids = (torch.arange(m, device="cuda") % 8).int()
    clean = L.loract_lora_requests(x, a, b, ids, scales, residual=res)
    _check(clean, x, a, b, ids, scales, res)
    a[2, 5, 3], b[3, 1, 7], x[9, 0], scales[6], res[12, 4], x[21, 199] = NAN, INF, NAN, INF, NAN, INF
    got = L.loract_lora_requests(x, a, b, ids, scales, residual=res)
    token = torch.arange(m, device="cuda")
    own = (token == 9) | (token == 12) | (token == 21)
    untouched = ~((ids == 2) | (ids == 3) | (ids == 6) | own)
    assert torch.equal(got[untouched], clean[untouched]) and untouched.sum() > m // 2
    assert torch.isnan(got[ids == 2]).all() and torch.isnan(got[9]).all() and not torch.isfinite(got[ids == 6]).any() and not torch.isfinite(got[21]).any()
    row = (ids == 3) & ~own
    assert torch.isinf(got[row][:, 7]).all() and torch.equal(got[row][:, :7], clean[row][:, :7]) and torch.equal(got[row][:, 8:], clean[row][:, 8:])
    assert torch.isnan(got[12, 4]) and torch.equal(got[12, :4], clean[12, :4]) and torch.equal(got[12, 5:], clean[12, 5:])
