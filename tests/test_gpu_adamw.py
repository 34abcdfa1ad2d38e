"""AdamW over many tensors against the formulas in 64 bits.

Bounds.  m' and v' are sums of two products whose factors (constants, and in v' the square) are rounded: at most four roundings of
float32 each way, 4 2^-24 of the terms' magnitudes.  p' adds about ten (m', v' and the root with theirs, the two rates, a sum, a quotient, a
product) on the move and three on p: 12 2^-24 of their magnitudes, and m's error, which is relative to its terms and not to their sum, as it is
multiplied.  An 8-bit code lies between those of the two ends of its moment's interval; so does a bf16 parameter.
"""
import numpy as np
import pytest
import torch

import paper_2509_23472_amd as L
import step_ref as ref

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
HYPER = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
SIZES = [[1], [255, 256, 257], [8, 0, 2048, 2049, 1, 4096 + 13], [31, 33, 7] * 40, [70000]]


def _make(sizes, p_dtype, g_dtype, seed, offset=0):
    """Tensors that begin `offset` elements into their memory."""
    gen = torch.Generator().manual_seed(seed)

    def tensors(dtype, scale):
        out = []
        for n in sizes:
            t = torch.empty(n + offset, dtype=dtype, device="cuda")[offset:]
            t.copy_(torch.randn(n, generator=gen) * scale)
            out.append(t)
        return out
    return tensors(p_dtype, 0.1), tensors(g_dtype, 1e-2)


def _flat(ts):
    return np.concatenate([t.double().cpu().numpy() for t in ts]) if ts else np.zeros(0)


def _held(state, place):
    """(m, v) of the tensors' elements in 64 bits."""
    if state.bits == 32:
        return state.m.double().cpu().numpy()[place], state.v.double().cpu().numpy()[place]
    unit = np.exp2(state.exps.cpu().numpy().astype(np.float64) - 127).repeat(ref.BLOCK, 0)
    return (state.m.double().cpu().numpy() * unit[:, 0])[place], ((state.v.double().cpu().numpy() * unit[:, 1]) ** 2)[place]


def _check_codes(codes, exps, want, off, bits, place, what):
    """codes, exps: what the step stored; want +- off: the moments (or roots) in 64 bits; bits: 10 of each element."""
    total = len(codes)
    lo, hi = np.zeros(total), np.zeros(total)
    lo[place], hi[place] = np.maximum(np.abs(want) - off, 0), np.abs(want) + off
    for b in range(total // ref.BLOCK):
        sl = slice(b * ref.BLOCK, (b + 1) * ref.BLOCK)
        byte = int(exps[b])
        assert ref.unit_byte(lo[sl].max()) <= byte <= ref.unit_byte(hi[sl].max()), (what, b)
        unit = 2.0 ** (byte - 127)
        least, most = (ref.rounded(x[sl] / unit, bits[sl], 10, 3, -6) for x in (lo, hi))
        if what == "root":
            least, most = (np.where(x[sl] > 0, np.maximum(y, 2.0 ** -9), y) for x, y in ((lo, least), (hi, most)))
        got = np.abs(codes[sl])
        assert (got >= least).all() and (got <= most).all(), (what, b, got, least, most)


def _step_and_check(params, grads, state, sizes, step, seed, copies=None, grad_scale=None, **kw):
    h = dict(HYPER, **kw)
    place, scale = ref.places(sizes), 1.0 if grad_scale is None else float(grad_scale)
    m0, v0 = _held(state, place)
    p0, g0 = _flat(params), _flat(grads) * scale
    L.loract_adamw(params, grads, state, step=step, seed=seed, copies=copies, grad_scale=grad_scale, **h)
    torch.cuda.synchronize()
    b1, b2 = h["betas"]
    p, m, v, size = ref.adamw(p0, g0, m0, v0, step, h["lr"], h["betas"], h["eps"], h["weight_decay"])
    off_m = 5 * U32 * (b1 * np.abs(m0) + (1 - b1) * np.abs(g0))        # (a fifth: grad_scale)
    off_v = 7 * U32 * v                                               # (two more for it)
    den = np.sqrt(v) / np.sqrt(1 - b2 ** step) + h["eps"]
    off_p = 14 * U32 * size + h["lr"] / (1 - b1 ** step) * off_m / den
    got_p = _flat(params)
    words = ref.halves(seed, step, len(state.m)) if len(state.m) < 30000 else None
    if params[0].dtype is torch.float32:
        assert (np.abs(got_p - p) <= off_p).all(), np.abs(got_p - p).max()
    elif words is not None:
        lo, hi = (ref.rounded(x, (words >> 20)[place], 12, 7, -126) for x in (np.maximum(np.abs(p) - off_p, 0), np.abs(p) + off_p))
        assert (np.abs(got_p) >= lo).all() and (np.abs(got_p) <= hi).all()
    else:
        assert (np.abs(got_p - p) <= 2.0 ** -7 * np.abs(p) + off_p).all()         # a random rounding is off by less than a spacing
    if copies is not None:
        assert all(torch.equal(c, q.bfloat16()) for c, q in zip(copies, params))
    if state.bits == 32:
        got_m, got_v = _held(state, place)
        assert (np.abs(got_m - m) <= off_m).all() and (np.abs(got_v - v) <= off_v).all()
    elif words is not None:
        codes_m, codes_r = state.m.double().cpu().numpy(), state.v.double().cpu().numpy()
        exps = state.exps.cpu().numpy()
        assert (np.sign(codes_m[place]) * np.sign(m) >= 0).all() and (codes_r >= 0).all()
        _check_codes(codes_m, exps[:, 0], m, off_m, words & 1023, place, "m")
        _check_codes(codes_r, exps[:, 1], np.sqrt(v), 5 * U32 * np.sqrt(v), (words >> 10) & 1023, place, "root")


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s[:4])))
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                             (torch.float32, torch.bfloat16)])
def test_three_steps(sizes, bits, p_dtype, g_dtype):
    params, grads = _make(sizes, p_dtype, g_dtype, 1)
    state = L.loract_adamw_state(params, bits=bits)
    for step in (1, 2, 3):
        _step_and_check(params, grads, state, sizes, step, 77)
        for g in grads:
            g.mul_(-0.7)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 3])
def test_tensors_at_any_address_with_copies_and_scale(bits, offset):
    sizes = [511, 8, 4100, 3]
    params, grads = _make(sizes, torch.float32, torch.bfloat16, 2, offset)
    copies = [torch.full((n + 1,), 7.0, dtype=torch.bfloat16, device="cuda")[1:] for n in sizes]
    state = L.loract_adamw_state(params, bits=bits)
    scale = torch.tensor([0.37], device="cuda")
    for step in (1000, 1001):
        _step_and_check(params, grads, state, sizes, step, 2 ** 64 - 5, copies=copies, grad_scale=scale)


def test_nothing_is_written_outside_the_tensors():
    sizes = [5, 300, 2047]
    flat = torch.full((4096,), 3.0, device="cuda")
    at = [10, 100, 1000]
    params = [flat[a:a + n] for a, n in zip(at, sizes)]
    grads = [torch.ones(n, device="cuda") for n in sizes]
    L.loract_adamw(params, grads, L.loract_adamw_state(params, bits=8), step=1, **HYPER)
    inside = torch.zeros(4096, dtype=torch.bool)
    for a, n in zip(at, sizes):
        inside[a:a + n] = True
    got = flat.cpu()
    assert (got[~inside] == 3.0).all() and (got[inside] != 3.0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_gradients_and_moments(bits):
    params, _ = _make([700], torch.float32, torch.float32, 3)
    before = params[0].clone()
    state = L.loract_adamw_state(params, bits=bits)
    L.loract_adamw(params, [torch.zeros_like(params[0])], state, step=1, **dict(HYPER, weight_decay=0.0))
    assert torch.equal(params[0], before) and (state.m.float() == 0).all() and (state.v.float() == 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_with_its_element(bits, bad):
    """The other elements of a block keep their values."""
    params, grads = _make([600], torch.float32, torch.float32, 4)
    clean, other = params[0].clone(), L.loract_adamw_state(params, bits=bits)
    state = L.loract_adamw_state(params, bits=bits)
    L.loract_adamw([clean], grads, other, step=1, **HYPER)
    grads[0][300] = bad
    L.loract_adamw(params, grads, state, step=1, **HYPER)
    keep = torch.arange(600, device="cuda") != 300
    assert torch.isnan(params[0][300]) and torch.equal(params[0][keep], clean[keep])
    assert not torch.isfinite(state.m.float()[300]) and not torch.isfinite(state.v.float()[300])
    far = torch.ones(768, dtype=torch.bool, device="cuda")
    far[300] = False
    if bits == 32:
        assert torch.equal(state.m[far], other.m[far])
    else:
        # the block's unit may follow its other elements only: theirs are the codes of a block without this one
        unit = torch.exp2(state.exps.double() - 127).repeat_interleave(256, 0)
        unit_other = torch.exp2(other.exps.double() - 127).repeat_interleave(256, 0)
        near = torch.zeros(768, dtype=torch.bool, device="cuda")
        near[256:512] = True
        assert torch.equal(state.m.double()[far & ~near], other.m.double()[far & ~near])
        a, b = (state.m.double() * unit[:, 0])[far & near], (other.m.double() * unit_other[:, 0])[far & near]
        assert ((a - b).abs() <= b.abs() / 4 + unit_other[256, 0] / 256).all()


def test_extreme_magnitudes_in_8_bits():
    for scale in (1e-30, 1e-18, 1.0, 1e17):
        params, grads = _make([512], torch.float32, torch.float32, 5)
        grads[0].mul_(scale)
        grads[0][:7] *= 1e-6
        state = L.loract_adamw_state(params, bits=8)
        # v = 0.001 g^2 is zero in float32 for |g| below 2^-149.5 / sqrt(0.001) ~ 1e-21: the smallest gradients, 1e-6 1e-2 scale, need an eps
        # unless scale is above 1e-12 or so, by the formula itself
        held = scale > 1e-12
        for s in (1, 2):
            L.loract_adamw(params, grads, state, step=s, **dict(HYPER, eps=0.0 if held else 1e-8))
        assert torch.isfinite(params[0]).all() and torch.isfinite(state.m.float()).all()
        assert not held or (state.v.float()[:512] > 0).all()


def test_random_rounding_is_right_on_average():
    """m = 1.03125 beside the largest element: a quarter of the way from 1 to its neighbour.  Of 2^16 independent roundings a quarter goes up, within six
    deviations, sqrt(2^16 3/16) each."""
    n = 1 << 16
    g = torch.full((n,), 1.03125, device="cuda")
    params = [torch.zeros(n, device="cuda")]
    ups = []
    for seed in (1, 2):
        state = L.loract_adamw_state(params, bits=8)
        L.loract_adamw(params, [g], state, step=1, lr=0.0, betas=(0.0, 0.0), weight_decay=0.0, seed=seed)
        value = state.m.double() * torch.exp2(state.exps[:, 0].double() - 127).repeat_interleave(256)
        assert ((value == 1.0) | (value == 1.125)).all()
        ups.append(value == 1.125)
        assert abs(int(ups[-1].sum()) - n / 4) <= 6 * (n * 3 / 16) ** 0.5
    assert not torch.equal(*ups)


def test_equal_calls_give_equal_bits_and_steps_differ():
    def run(step):
        params, grads = _make([5000, 33], torch.bfloat16, torch.float32, 6)
        state = L.loract_adamw_state(params, bits=8)
        L.loract_adamw(params, grads, state, step=step, seed=9, **HYPER)
        return params + [state.m.view(torch.uint8), state.v.view(torch.uint8), state.exps]
    a, b, c = run(5), run(5), run(6)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and not torch.equal(a[2], c[2])


def test_many_tensors_take_several_launches():
    sizes = [17 + i % 5 for i in range(333)]
    params, grads = _make(sizes, torch.float32, torch.float32, 7)
    _step_and_check(params, grads, L.loract_adamw_state(params), sizes, 1, 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_takes_rate_step_and_scale_from_the_device(bits):
    sizes = [300, 4099]
    params, grads = _make(sizes, torch.bfloat16, torch.float32, 8)
    eager = [p.clone() for p in params]
    state, other = L.loract_adamw_state(params, bits=bits), L.loract_adamw_state(params, bits=bits)
    lr, step, scale = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.loract_adamw(params, grads, state, step=step, lr=lr, grad_scale=scale, seed=3)
    rates = [2.0 ** -7, 2.0 ** -8, 2.0 ** -9, 2.0 ** -8]
    for i, rate in enumerate(rates):
        lr.fill_(rate)
        step.fill_(i + 1)
        scale.fill_(1.0 / (i + 1))
        graph.replay()
        L.loract_adamw(eager, [g * scale for g in grads], other, step=i + 1, lr=rate, seed=3)
        torch.cuda.synchronize()
        # the two form 1 - beta^t by another function: 2^-24 of the rate, which a random rounding may turn into a spacing now and then
        for a, b in zip(params, eager):
            assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs()).all() and (a != b).float().mean() < 1e-2
        for a, b in zip(params, eager):
            b.copy_(a)
        assert torch.equal(state.m.view(torch.uint8), other.m.view(torch.uint8)) and torch.equal(state.v.view(torch.uint8), other.v.view(torch.uint8))


def test_another_stream():
    params, grads = _make([100000], torch.float32, torch.float32, 9)
    state = L.loract_adamw_state(params)
    want = [p.clone() for p in params]
    L.loract_adamw(want, grads, L.loract_adamw_state(want), step=1, **HYPER)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.loract_adamw(params, grads, state, step=1, **HYPER)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(params[0], want[0])
