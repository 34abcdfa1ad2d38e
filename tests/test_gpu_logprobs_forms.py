"""The forms of the log probabilities' kernels that a vocabulary's size and the number of rows choose, each with its first and last size; logits of the type's
lowest value; against the formulas in 64 bits with the bounds of test_gpu_logprobs.py."""
import pytest
import torch

import paper_2509_23472_amd as L
import step_ref as ref
from test_gpu_logprobs import BF, F32, INF, U, _bound, _check_forward, _check_grad, _close, _logits

pytestmark = pytest.mark.gpu


def _few(m):
    return torch.unique(torch.tensor([0, 1, 2, m // 2, m - 2, m - 1], device="cuda"))


# Rows of a workgroup's registers: 16-byte pieces up to 512, 2048, 4096, 8192, 16384, and behind them rows of which the rest is read again.
HELD = [(pieces, extra) for pieces in (2, 512, 2048, 4096, 8192, 16384, 32767) for extra in (0, 1, 3)]


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("pieces,extra", HELD)
def test_both_in_one_call_of_every_length(pieces, extra, dtype, entropy):
    """`extra` 0 and 3: the last sizes of a form (with a few elements around the whole pieces, rows that start anywhere); 1: the first of the next."""
    m, each = 130, 8 if dtype is BF else 4
    n = pieces * each + (each if extra == 1 else extra)
    x, t, gen = _logits(m, n, dtype, pieces + extra, pad=extra)
    t[5:9] = -1
    x[3, n // 2:] = -INF
    d_logp = torch.randn(m, generator=gen, device="cuda")
    d_entropy = torch.randn(m, generator=gen, device="cuda") if entropy else None
    before = x.clone()
    logp, h, grad = L.loract_token_logprobs_grad(x, t, d_logp, d_entropy)
    assert torch.equal(x, before) and (grad[5:9] == 0).all() != entropy
    rows = _few(m)
    rows = torch.cat([rows, torch.tensor([3, 5], device="cuda")])
    _check_grad(grad[rows], x[rows], t[rows], d_logp[rows], None if d_entropy is None else d_entropy[rows])
    _, _, want_h, want = ref.logprobs(x[rows], t[rows])
    b = _bound(x[rows], 1.0)
    _close(logp[rows], want, b + 60 * U, "logp")
    _close(h[rows], want_h, 4 * b * want_h.clamp(min=1), "entropy")
    whole = x._base.clone()
    again = whole[:, :n]
    L.loract_token_logprobs_grad(again, t, d_logp, d_entropy, out=again)
    assert torch.equal(again, grad) and torch.equal(whole[:, n:], x._base[:, n:])


@pytest.mark.parametrize("m,n,dtype", [(128, 50257, BF), (300, 128256, BF), (200, 32000, F32), (127, 50257, BF), (127, 128256, F32)])
def test_vocabularies_in_use(m, n, dtype):
    x, t, gen = _logits(m, n, dtype, 21)
    d_logp, d_entropy = (torch.randn(m, generator=gen, device="cuda") for _ in range(2))
    rows = _few(m)
    for dl, de in ((d_logp, None), (d_logp, d_entropy), (None, d_entropy)):
        grad = L.loract_token_logprobs_grad(x, t, dl, de, temperature=0.7)[2]
        _check_grad(grad[rows], x[rows], t[rows], None if dl is None else dl[rows], None if de is None else de[rows], 0.7)
    f = _check_forward(x[rows], t[rows], 0.7, top=20)
    whole = L.loract_token_logprobs(x, t, temperature=0.7, top=20)
    assert torch.equal(whole.top_ids[rows], f.top_ids)


@pytest.mark.parametrize("temperature", [1.0, 2.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,n", [(6, 300), (6, 40000), (600, 4099), (150, 140003)])
def test_targets_that_have_the_lowest_value(m, n, dtype, temperature):
    """A mask of the type's lowest value beside other logits: log p of what it masks is that value / T less the row's, and finite."""
    x, t, gen = _logits(m, n, dtype, 22)
    low = torch.finfo(dtype).min
    x[:4, 2:] = low
    t[:4] = n - 1
    x[4, ::2] = low
    t[4] = 0
    rows = torch.tensor([0, 1, 3, 4, 5], device="cuda")
    log_p, _, entropy, want = ref.logprobs(x[rows], t[rows], temperature)
    assert torch.isfinite(want).all()
    b = _bound(torch.where(x[rows] > low, x[rows], torch.zeros_like(x[rows])), temperature)

    def off(v, b):
        # far values: three roundings (x - M, 1 / T, their product) and that of the last difference, relative to log p
        return torch.where(v < -1e30, 4 * U * v.abs(), b + 60 * U)
    f = L.loract_token_logprobs(x, t, temperature=temperature, top=5)
    _close(f.logp[rows], want, off(want, b), "logp")
    _close(f.entropy[rows], entropy, 4 * b * entropy.clamp(min=1), "entropy")
    assert torch.equal(f.top_ids[rows], ref.top(x[rows], 5))
    ranked = log_p.gather(1, f.top_ids[rows].long())
    _close(f.top_logp[rows], ranked, off(ranked, b[:, None]), "top_logp")
    one = torch.ones(m, device="cuda")
    logp, _, grad = L.loract_token_logprobs_grad(x, t, one, temperature=temperature)
    _close(logp[rows], want, off(want, b), "logp")
    g, size = ref.logprobs_grad(x[rows], t[rows], one[rows], None, temperature)
    unit = 2.0 ** -8 if dtype is BF else U
    for got in (grad, L.loract_token_logprobs_backward(x, t, f.stats, one, temperature=temperature)):
        _close(got[rows], g, 2 * b[:, None] * size + unit * g.abs() + 2.0 ** -126, "gradient")
