"""Log probabilities, entropy, alternatives and their gradients against the formulas in 64 bits.

Bounds, in units of U = 2^-24.  x / T and t = x / T - M: a rounding each of the factor 1 / T and of the result, 2 U (|x / T| + |t|), which e^t
carries as a relative error; the exponential itself: |t| 2^-23 + 4 U for bf16 logits, 4 U for float32.  With R = max |x| / T and terms beyond t = -30 below
rounding, a term of S is off by e = 2 U (R + 30) + 60 U + 4 U of itself at most, and so are S and W (the running maximum multiplies by at most one more
such factor for each of its few new values: 3 e in all; sums of n positive terms by lanes and trees: 6 sqrt(n) U).  log p then is off by that and its own
roundings, 3 U (|log p| + R); the entropy, log S - W / S, by four times that relative to max(1, H).
"""
import math

import pytest
import torch

import paper_2509_23472_amd as L
import step_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def _bound(x, t):
    r = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).float().abs().amax(1).double() / t
    return 3 * (2 * U * (r + 30) + 64 * U) + 6 * math.sqrt(x.shape[1]) * U


def _logits(m, n, dtype, seed=0, scale=3.0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(m, n + pad, generator=gen, device="cuda").mul_(scale).to(dtype)[:, :n]
    t = torch.randint(0, n, (m,), generator=gen, device="cuda")
    return x, t, gen


def _close(got, want, bound, what):
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got.double() - want).abs() <= bound))
    assert not bad.any(), (what, bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


def _check_forward(x, targets, temperature=1.0, top=0):
    f = L.loract_token_logprobs(x, targets, temperature=temperature, top=top)
    log_p, _, entropy, logp = ref.logprobs(x, targets, temperature)
    b = _bound(x, temperature)
    r = torch.where(torch.isfinite(x), x, torch.zeros_like(x)).float().abs().amax(1).double() / temperature
    if targets is not None:
        _close(f.logp, logp, b + 3 * U * (torch.nan_to_num(logp, neginf=0.0).abs() + r), "logp")
    _close(f.entropy, entropy, 4 * b * entropy.clamp(min=1), "entropy")
    if top:
        ids = ref.top(x, top)
        assert torch.equal(f.top_ids, ids)
        want = log_p.gather(1, ids.long())
        _close(f.top_logp, want, (b + 3 * U * r)[:, None] + 3 * U * torch.nan_to_num(want, neginf=0.0).abs(), "top_logp")
    else:
        assert f.top_ids is None and f.top_logp is None
    return f


def _check_grad(got, x, targets, d_logp, d_entropy, temperature=1.0, refined_extra=0.0):
    want, size = ref.logprobs_grad(x, targets, d_logp, d_entropy, temperature)
    b = _bound(x, temperature)
    # p carries e and S's error, log p + H the absolute errors of both: the terms' sizes count what is multiplied, p (1 + |t|) b more what is added
    _, p, entropy, _ = ref.logprobs(x, targets, temperature)
    extra = 0.0 if d_entropy is None else d_entropy.double().abs()[:, None] * p * (6 * b * entropy.clamp(min=1))[:, None] / temperature
    unit = 2.0 ** -8 if x.dtype is BF else U
    # an exponential below 2^-126 is zero: p loses 2^-126 at most (S >= 1), and p |log p|, which grows with p there, 2^-126 (88 + log S + 1)
    lost = (0.0 if d_logp is None else d_logp.double().abs()) + (0.0 if d_entropy is None else d_entropy.double().abs() * (100 + entropy))
    lost = 2.0 ** -126 * lost[:, None] / temperature
    _close(got, want, 2 * b[:, None] * size + extra + lost + unit * torch.nan_to_num(want).abs() + 2.0 ** -133, "gradient")


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 64), (7, 255), (4, 1000), (3, 4097), (2, 32000), (1, 50257), (300, 511), (700, 2050)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("m,n", SHAPES)
def test_forward_and_gradients(m, n, dtype):
    x, t, gen = _logits(m, n, dtype, m * n, pad=3)
    t[::3] = -1
    d_logp, d_entropy = (torch.randn(m, generator=gen, device="cuda") for _ in range(2))
    f = _check_forward(x, t, top=min(n, 5))
    for dl, de in ((d_logp, None), (d_logp, d_entropy), (None, d_entropy)):
        _check_grad(L.loract_token_logprobs_backward(x, t, f.stats, dl, de), x, t, dl, de)
        logp, entropy, grad = L.loract_token_logprobs_grad(x, t, dl, de)
        _check_grad(grad, x, t, dl, de)
        b = _bound(x, 1.0)
        _close(logp, ref.logprobs(x, t)[3], b + 40 * U, "logp")
        _close(entropy, ref.logprobs(x, t)[2], 4 * b * ref.logprobs(x, t)[2].clamp(min=1), "entropy")


@pytest.mark.parametrize("m,n,dtype", [(600, 17000, BF), (520, 33000, F32), (513, 70001, F32), (515, 140000, BF), (400, 131001, F32), (130, 300000, BF), (130, 131100, F32), (1030, 32000, BF), (600, 4100, F32)])
def test_rows_in_registers_and_rows_that_are_too_long(m, n, dtype):
    x, t, gen = _logits(m, n, dtype, 5)
    d_logp = torch.randn(m, generator=gen, device="cuda")
    d_entropy = torch.randn(m, generator=gen, device="cuda")
    logp, entropy, grad = L.loract_token_logprobs_grad(x, t, d_logp, d_entropy)
    rows = torch.tensor([0, 1, 2, 3, m // 2, m - 2, m - 1], device="cuda")
    _check_grad(grad[rows], x[rows], t[rows], d_logp[rows], d_entropy[rows])
    _close(logp[rows], ref.logprobs(x[rows], t[rows])[3], _bound(x[rows], 1.0) + 60 * U, "logp")
    _check_forward(x[rows], t[rows])


@pytest.mark.parametrize("temperature", [0.05, 0.7, 3.0])
@pytest.mark.parametrize("targets", [torch.int32, torch.int64])
def test_temperature_and_types_of_targets(temperature, targets):
    x, t, gen = _logits(9, 3001, F32, 3)
    t = t.to(targets)
    d_logp, d_entropy = (torch.randn(9, generator=gen, device="cuda") for _ in range(2))
    f = _check_forward(x, t, temperature, top=20)
    _check_grad(L.loract_token_logprobs_backward(x, t, f.stats, d_logp, d_entropy, temperature=temperature), x, t, d_logp, d_entropy, temperature)
    _check_grad(L.loract_token_logprobs_grad(x, t, d_logp, d_entropy, temperature=temperature)[2], x, t, d_logp, d_entropy, temperature)


@pytest.mark.parametrize("m", [1, 20, 600])
@pytest.mark.parametrize("n", [70, 9000])
@pytest.mark.parametrize("top", [1, 2, 63, 64])
def test_alternatives_with_ties(m, n, top):
    """bf16 logits of few values: many ties."""
    x, t, gen = _logits(m, n, BF, top, scale=1.0)
    x = (x * 2).round() / 2
    _check_forward(x, t, top=top)


@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "zeros", "mostly ruled out", "one left"])
@pytest.mark.parametrize("m,n", [(2, 70000), (600, 5000), (3, 65)])
def test_alternatives_of_awkward_rows(kind, m, n):
    x = torch.zeros(m, n, device="cuda")
    if kind in ("rising", "falling"):
        x = torch.arange(n, device="cuda").float().repeat(m, 1) * (1e-3 if kind == "rising" else -1e-3)
    if kind == "zeros":
        x[:, ::2] = -0.0
    if kind == "mostly ruled out":
        x.fill_(-INF)
        x[:, 7::41] = 1.0
    if kind == "one left":
        x.fill_(-INF)
        x[:, n - 1] = 2.0
    _check_forward(x, torch.full((m,), n - 1, device="cuda"), top=50)


@pytest.mark.parametrize("dtype,trip", [(BF, 2048), (F32, 1024)])
@pytest.mark.parametrize("m", [2, 600])
def test_clumped_maxima_exceed_the_candidates(m, dtype, trip):
    """All large elements lie where 63 of a workgroup's 256 threads read in every trip: the 64th largest of the threads' maxima is small, and
    thousands of elements lie above it."""
    x = torch.zeros(m, 60000, device="cuda")
    for j in range(60000 // trip):
        x[:, trip * j:trip * j + 63 * trip // 256] = 10.0 + (j * 7) % 50
    x[:, 59000] = 100.0
    _check_forward(x.to(dtype), None, top=64)


def test_masked_rows_and_lowest_values():
    for dtype in (BF, F32):
        for m, n in ((6, 300), (6, 40000), (600, 4099), (150, 140003)):
            x, t, gen = _logits(m, n, dtype, 8)
            x[0] = -INF                                    # nothing is left
            x[1] = torch.finfo(dtype).min                  # the type's lowest value everywhere: as good as equal
            x[2, 1:] = -INF                                # one token is left, the target another
            t[2] = n - 1
            x[3, ::2] = torch.finfo(dtype).min
            x[4, 3:] = -INF
            t[4] = 1
            d_logp, d_entropy = torch.ones(m, device="cuda"), torch.full((m,), 0.5, device="cuda")
            f = L.loract_token_logprobs(x, t, top=4)
            log_p, p, entropy, logp = ref.logprobs(x, t)
            assert f.logp[0] == -INF and f.entropy[0] == 0 and (f.top_logp[0] == -INF).all() and f.top_ids[0].tolist() == [0, 1, 2, 3]
            assert f.logp[2] == -INF and f.entropy[2] == 0 and f.top_logp[2].tolist() == [0.0, -INF, -INF, -INF]
            few = slice(0, 6)
            keep = torch.tensor([1, 2, 4, 5], device="cuda")
            _close(f.logp[keep], logp[keep], 1e-5, "logp")
            _close(f.entropy[few], entropy[few], 1e-4, "entropy")
            assert torch.equal(f.top_ids[few], ref.top(x[few], 4))
            for grad in (L.loract_token_logprobs_backward(x, t, f.stats, d_logp, d_entropy), L.loract_token_logprobs_grad(x, t, d_logp, d_entropy)[2]):
                want = ref.logprobs_grad(x[few], t[few], d_logp[few], d_entropy[few])[0]
                assert (grad[0] == 0).all() and torch.isfinite(grad[few]).all()
                unit = 2.0 ** -8 if dtype is BF else 1e-5          # (half a step of bf16 is 2^-8 of the value)
                assert ((grad[few].double() - want).abs() <= unit * want.abs() + 1e-5).all()


def test_what_is_no_number_and_targets_out_of_range():
    for m, n in ((5, 700), (5, 20000), (600, 5000), (150, 80000)):
        x, t, _ = _logits(m, n, F32, 9)
        clean = L.loract_token_logprobs(x, t, top=3)
        x[0, 5] = float("nan")
        x[1, 6] = INF
        t[2] = n
        t[3] = 2 ** 40
        f = L.loract_token_logprobs(x, t, top=3)
        assert torch.isnan(f.logp[:4]).all() and torch.isnan(f.entropy[:2]).all() and torch.isnan(f.top_logp[:2]).all()
        assert torch.equal(f.entropy[2:], clean.entropy[2:]) and torch.equal(f.logp[4:], clean.logp[4:])
        assert torch.equal(f.top_ids[0], ref.top(x[:1], 3)[0]) and f.top_ids[1, 0] == 6
        one = torch.ones(m, device="cuda")
        want = L.loract_token_logprobs_backward(x[4:], t[4:], L.loract_token_logprobs(x[4:], t[4:]).stats, one[4:])
        for grad in (L.loract_token_logprobs_backward(x, t, f.stats, one), L.loract_token_logprobs_grad(x, t, one)[2]):
            assert torch.isnan(grad[:4]).all() and torch.isfinite(grad[4:]).all()
            assert (grad[4:] - want).abs().max() <= 1e-6
        t[:] = -1                                             # no target: no gradient, whatever the row holds
        assert (L.loract_token_logprobs_backward(x, t, f.stats, one) == 0).all() and (L.loract_token_logprobs_grad(x, t, one)[2] == 0).all()


@pytest.mark.parametrize("m,n,dtype", [(600, 5000, BF), (3, 20001, BF), (700, 3001, F32), (200, 80003, F32)])
def test_in_place_and_strided(m, n, dtype):
    x, t, gen = _logits(m, n, dtype, 10, pad=5)
    d = torch.randn(m, generator=gen, device="cuda")
    f = L.loract_token_logprobs(x, t)
    want = L.loract_token_logprobs_backward(x, t, f.stats, d)
    memory = torch.full((m, n + 9), 7.0, dtype=dtype, device="cuda")
    out = memory[:, 2:n + 2]
    assert torch.equal(L.loract_token_logprobs_backward(x, t, f.stats, d, out=out), want) and (memory[:, :2] == 7).all() and (memory[:, n + 2:] == 7).all()
    logp, _, one = L.loract_token_logprobs_grad(x, t, d)
    memory.fill_(7.0)
    assert torch.equal(L.loract_token_logprobs_grad(x, t, d, out=out)[2], one) and (memory[:, :2] == 7).all() and (memory[:, n + 2:] == 7).all()
    whole = x._base.clone()
    again = whole[:, :n]
    got = L.loract_token_logprobs_grad(again, t, d, out=again)
    assert torch.equal(again, one) and torch.equal(got[0], logp) and torch.equal(whole[:, n:], x._base[:, n:])
    again = x._base.clone()[:, :n]
    L.loract_token_logprobs_backward(again, t, f.stats, d, out=again)
    assert torch.equal(again, want)


def test_gradient_against_differences():
    """Central differences of the forward call in float32: steps of 2^-5 leave a relative error of 2^-10 / 6 times third derivatives of at most
    one, and 2 2^-22 / 2^-4 of the values' roundings."""
    x, t, gen = _logits(4, 50, F32, 11, scale=1.0)
    d_logp, d_entropy = (torch.randn(4, generator=gen, device="cuda") for _ in range(2))
    grad = L.loract_token_logprobs_grad(x, t, d_logp, d_entropy, temperature=1.5)[2]
    step = 2.0 ** -5
    for j in (0, 7, 49, int(t[0])):
        ends = []
        for sign in (1, -1):
            y = x.clone()
            y[:, j] += sign * step
            f = L.loract_token_logprobs(y, t, temperature=1.5)
            ends.append(f.logp.double() * d_logp + f.entropy.double() * d_entropy)
        slope = (ends[0] - ends[1]) / (2 * step)
        assert ((slope - grad[:, j]).abs() <= 6 * step ** 2 + 1e-4).all()


def test_empty_and_equal_calls():
    f = L.loract_token_logprobs(torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)
    assert f.logp.shape == (0,) and f.top_ids.shape == (0, 2)
    assert L.loract_token_logprobs_grad(torch.zeros(0, 10, device="cuda"), None, None, torch.zeros(0, device="cuda"))[2].shape == (0, 10)
    x, t, _ = _logits(33, 30011, BF, 12)
    a, b = (L.loract_token_logprobs(x, t, top=64) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_captured_calls_beside_eager_ones():
    x, t, gen = _logits(40, 33000, BF, 13)
    d = torch.randn(40, generator=gen, device="cuda")
    L.loract_token_logprobs(x, t, top=8)
    torch.cuda.synchronize()
    graphs = []
    for top in (8, 3):                                   # two graphs: each has a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f = L.loract_token_logprobs(x, t, top=top)
            g = L.loract_token_logprobs_grad(x, t, d)
        graphs.append((graph, f, g))
    for i in range(4):
        x.copy_(torch.randn(40, 33000, generator=gen, device="cuda"))
        for graph, _, _ in graphs:
            graph.replay()
        want = L.loract_token_logprobs(x, t, top=8)
        grad = L.loract_token_logprobs_grad(x, t, d)
        torch.cuda.synchronize()
        for (_, f, g), top in zip(graphs, (8, 3)):
            assert torch.equal(f.logp, want.logp) and torch.equal(f.top_ids, want.top_ids[:, :top]) and torch.equal(f.top_logp, want.top_logp[:, :top])
            assert all(torch.equal(p, q) for p, q in zip(g, grad))


def test_another_stream():
    x, t, _ = _logits(64, 32000, BF, 14)
    want = L.loract_token_logprobs(x, t, top=5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = L.loract_token_logprobs(x, t, top=5)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("m,n", [(7, 20000), (600, 5000), (700, 140001)])
def test_entropy_without_targets(m, n):
    x, _, gen = _logits(m, n, BF, 15)
    d = torch.randn(m, generator=gen, device="cuda")
    f = L.loract_token_logprobs(x, top=3)
    assert f.logp is None and torch.equal(f.top_ids[:5], ref.top(x[:5], 3))
    few = slice(0, 9)
    _check_grad(L.loract_token_logprobs_backward(x, None, f.stats, None, d)[few], x[few], None, None, d[few])
    logp, entropy, grad = L.loract_token_logprobs_grad(x, None, None, d)
    assert logp is None
    _check_grad(grad[few], x[few], None, None, d[few])
    _close(entropy[few], ref.logprobs(x[few], None)[2], 4 * _bound(x[few], 1.0) * ref.logprobs(x[few], None)[2].clamp(min=1), "entropy")


@pytest.mark.parametrize("n,dtype", [(3, F32), (9, BF)])
def test_more_rows_than_a_launch_has(n, dtype):
    m = (1 << 20) + 77
    x, t, gen = _logits(m, n, dtype, 16)
    d = torch.randn(m, generator=gen, device="cuda")
    f = L.loract_token_logprobs(x, t, top=2)
    log_p, _, entropy, logp = ref.logprobs(x, t)
    b = _bound(x, 1.0)
    _close(f.logp, logp, b + 40 * U, "logp")
    _close(f.entropy, entropy, 4 * b * entropy.clamp(min=1), "entropy")
    assert torch.equal(f.top_ids[-100:], ref.top(x[-100:], 2))
    _check_grad(L.loract_token_logprobs_backward(x, t, f.stats, d), x, t, d, None)
    _check_grad(L.loract_token_logprobs_grad(x, t, d)[2], x, t, d, None)
