"""loract_qknorm_rope_forward and _backward against plain 64-bit arithmetic."""
import math

import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _table(n_pos, rot, theta=10000.0, first=0):
    angle = torch.arange(first, first + n_pos, dtype=torch.float64)[:, None] * theta ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return torch.stack([angle.cos(), angle.sin()], 1).float()


def _case(m, hq, hk, d, rot, dtype=torch.bfloat16, interleaved=False, gammas=True, positions=None, n_pos=None, layout="plain", seed=1):
    """layout: plain, packed (slices of one projection), heads (head-major), odd (unaligned slices)."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(seed)
    host = lambda h: torch.randn(m, h, d, generator=gen).mul_(1.5).to(dtype)
    q, k, dyq, dyk = host(hq), host(hk), host(hq), host(hk)
    gq, gk = ((1 + 0.3 * torch.randn(d, generator=gen)) for _ in range(2)) if gammas else (None, None)
    n_pos = n_pos or m
    table = _table(n_pos, rot) if rot else None
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32)

    def place(a, b):
        """a and b on the GPU, and empty tensors like them, in the layout."""
        if layout == "plain":
            make = lambda t: torch.empty(t.shape, dtype=dtype, device="cuda")
            return make(a), make(b)
        if layout == "heads":
            make = lambda t: torch.empty((t.shape[1], m, d), dtype=dtype, device="cuda").transpose(0, 1)
            return make(a), make(b)
        lead = 8 if layout == "packed" else 1
        row = torch.full((m, lead + (hq + 2 * hk) * d + (lead if layout == "odd" else 0)), float("nan"), dtype=dtype, device="cuda")
        return row[:, lead:lead + hq * d].view(m, hq, d), row[:, lead + hq * d:lead + (hq + hk) * d].view(m, hk, d)

    def put(a, b):
        x, y = place(a, b)
        x.copy_(a)
        y.copy_(b)
        return x, y

    g = lambda t: None if t is None else t.cuda()
    dd = lambda t: None if t is None else t.double()
    keys = hk > 0
    args = dict(positions=g(pos), eps=EPS, interleaved=interleaved)
    (qd, kd), (dyqd, dykd) = put(q, k), put(dyq, dyk)
    if not keys:
        kd, dykd, gk = None, None, None
    out = place(q, k)
    qo, ko = L.loract_qknorm_rope_forward(qd, kd, g(gq), g(gk), g(table), out=out, **args)
    back = place(q, k)
    dq, dk, dgq, dgk = L.loract_qknorm_rope_backward(qd, kd, g(gq), g(gk), g(table), dyqd, dykd, out=back, **args)
    u = ref.U[dtype]
    eps = float(torch.tensor(EPS))
    for x, dy, gamma, y, dx, dg, what in ((q, dyq, gq, qo, dq, dgq, "q"), (k, dyk, gk, ko, dk, dgk, "k")):
        if what == "k" and not keys:
            assert y is None and dx is None and dg is None
            continue
        want, bound = ref.qknorm(x.double(), dd(gamma), dd(table), pos, eps, interleaved)
        ref.check(y, want, bound + 1.01 * u * (want.abs() + bound), "forward of " + what)
        want, bound, wg, bg = ref.qknorm(x.double(), dd(gamma), dd(table), pos, eps, interleaved, dy.double())
        ref.check(dx, want, bound + 1.01 * u * (want.abs() + bound), "backward of " + what)
        if gamma is None:
            assert dg is None
        else:
            ref.check(dg, wg, bg, "gamma's gradient of " + what)
    return qo, ko, dq, dk, dgq, dgk


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (80, 80), (80, 40), (96, 96), (256, 256), (32, 32), (8, 4), (6, 6), (7, 4),
                                   (1, 0), (33, 32), (512, 512), (1000, 500), (128, 0), (40, 24)])
@pytest.mark.parametrize("m,hq,hk", [(1, 1, 1), (5, 4, 2), (37, 12, 3)])
def test_head_sizes(m, hq, hk, d, rot, interleaved, dtype):
    _case(m, hq, hk, d, rot, dtype, interleaved)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["packed", "heads", "odd"])
@pytest.mark.parametrize("m,hq,hk,d,rot", [(3, 8, 2, 128, 128), (70, 6, 6, 64, 64), (9, 5, 1, 80, 40)])
def test_layouts(m, hq, hk, d, rot, layout, dtype):
    _case(m, hq, hk, d, rot, dtype, layout=layout)


@pytest.mark.parametrize("m,hq,hk,d", [(3000, 8, 2, 64), (700, 32, 8, 128), (2, 40, 0, 128), (1, 64, 64, 64), (1500, 3, 1, 50)])
def test_more_tokens_and_heads(m, hq, hk, d):
    _case(m, hq, hk, d, d)
    _case(m, hq, hk, d, d, gammas=False)


@pytest.mark.parametrize("d", [128, 50])
def test_positions_and_padding(d):
    pos = [0, 5, 199, 199, -1, 3, -7, 100, -2147483648, 17]
    qo, ko, dq, dk, _, _ = _case(10, 4, 2, d, d, positions=pos, n_pos=200)
    for i, p in enumerate(pos):
        if p < 0:
            assert not any(t[i].any() for t in (qo, ko, dq, dk))
    _case(6, 2, 2, d, d, positions=[-1] * 6, n_pos=4)                    # nothing but padding: no gradient


@pytest.mark.parametrize("d", [64, 50])
def test_infinities_in_padding_add_nothing(d):
    import paper_2509_23472_amd as L
    x = torch.randn(4, 2, d, device="cuda")
    dy = torch.randn(4, 2, d, device="cuda")
    gamma, table = torch.ones(d, device="cuda"), _table(8, d).cuda()
    pos = torch.tensor([0, -1, 2, -1], dtype=torch.int32, device="cuda")
    want = L.loract_qknorm_rope_backward(x, None, gamma, None, table, dy, None, positions=pos)
    x[1], x[3], dy[1], dy[3] = float("nan"), float("inf"), float("inf"), float("nan")
    got = L.loract_qknorm_rope_backward(x, None, gamma, None, table, dy, None, positions=pos)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert not L.loract_qknorm_rope_forward(x, None, gamma, None, table, positions=pos)[0][[1, 3]].any()


@pytest.mark.parametrize("d", [64, 50])
def test_positions_past_the_table_give_nan(d):
    import paper_2509_23472_amd as L
    x = torch.randn(3, 2, d, device="cuda")
    pos = torch.tensor([0, 8, 7], dtype=torch.int32, device="cuda")
    y, _ = L.loract_qknorm_rope_forward(x, None, None, None, _table(8, d).cuda(), positions=pos)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 2]]).all()
    dx = L.loract_qknorm_rope_backward(x, None, None, None, _table(8, d).cuda(), x, None, positions=pos)[0]
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[[0, 2]]).all()


@pytest.mark.parametrize("d", [128, 30])
def test_rows_of_zeros(d):
    import paper_2509_23472_amd as L
    x, dy = torch.zeros(3, 2, d, device="cuda"), torch.randn(3, 2, d, device="cuda")
    table = _table(3, d).cuda()
    assert not L.loract_qknorm_rope_forward(x, None, None, None, table, eps=1e-6)[0].any()
    dx = L.loract_qknorm_rope_backward(x, None, None, None, table, dy, None, eps=1e-6)[0]
    want = ref.qknorm(x.double().cpu(), None, table.double().cpu(), None, 1e-6, False, dy.double().cpu())[0]
    ref.check(dx, want, 1e-5 * want.abs() + 1e-2 * 2.0 ** -20, "dx")


def test_in_place_on_a_side_stream_and_repeated():
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(2)
    q, k = torch.randn(500, 8, 128, generator=gen).bfloat16().cuda(), torch.randn(500, 2, 128, generator=gen).bfloat16().cuda()
    dq, dk = torch.randn(500, 8, 128, generator=gen).bfloat16().cuda(), torch.randn(500, 2, 128, generator=gen).bfloat16().cuda()
    gamma, table = torch.rand(128, generator=gen).cuda(), L.loract_rope_table(500, 128)
    want = L.loract_qknorm_rope_backward(q, k, gamma, gamma, table, dq, dk)
    fwd = L.loract_qknorm_rope_forward(q, k, gamma, gamma, table)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = L.loract_qknorm_rope_backward(q, k, gamma, gamma, table, dq, dk, out=(dq, dk))
        L.loract_qknorm_rope_forward(q, k, gamma, gamma, table, out=(q, k))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert torch.equal(q, fwd[0]) and torch.equal(k, fwd[1])


def test_outputs_that_overlap_are_refused():
    import paper_2509_23472_amd as L
    x = torch.zeros((4, 2, 64), device="cuda")
    for bad in (x[:1].expand(4, 2, 64), x[:, :1].expand(4, 2, 64), x[:, :, ::2], x[:, :1], x.double()):
        with pytest.raises(ValueError):
            L.loract_qknorm_rope_forward(x, None, None, None, None, out=(bad, None))


def test_no_tokens():
    import paper_2509_23472_amd as L
    x, gamma, table = torch.zeros((0, 2, 64), device="cuda"), torch.ones(64, device="cuda"), L.loract_rope_table(4, 64)
    assert L.loract_qknorm_rope_forward(x, x, gamma, gamma, table)[0].shape == (0, 2, 64)
    assert not L.loract_qknorm_rope_backward(x, x, gamma, gamma, table, x, x)[2].any()


def test_offsets_past_32_bits():
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(4)
    m, d = 2100, 64
    x = torch.randn(m, 2, d, generator=gen).bfloat16()
    big = torch.empty((m, 1 << 20), dtype=torch.bfloat16, device="cuda")[:, :2 * d].view(m, 2, d)
    big.copy_(x)
    table = L.loract_rope_table(m, d)
    y, _ = L.loract_qknorm_rope_forward(big, None, None, None, table)
    want, bound = ref.qknorm(x.double(), None, table.double().cpu(), None, float(torch.tensor(1e-6)), False)
    ref.check(y, want, bound + 1.01 * ref.U[torch.bfloat16] * (want.abs() + bound), "y")


@pytest.mark.parametrize("first,n_pos,rot,theta", [(0, 300, 128, 10000.0), (1 << 20, 7, 64, 500000.0), (0, 1, 2, 10000.0)])
def test_table(first, n_pos, rot, theta):
    import paper_2509_23472_amd as L
    got = L.loract_rope_table(n_pos, rot, theta, first)
    # one rounding to float32, and 2^-50 of the angle (its factors and their product in float64)
    angle = (first + n_pos) * 2.0 ** -50
    want = torch.arange(first, first + n_pos, dtype=torch.float64)[:, None] * theta ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    want = torch.stack([want.cos(), want.sin()], 1)
    ref.check(got, want, 2.0 ** -24 + angle, "table")


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_against_differences(interleaved):
    """float32; every output's third derivative along unit directions is of order 1, its rounding 2^-22 |y| / h."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(6)
    m, heads, d, h = 12, 3, 64, 2.0 ** -6
    rand = lambda *s: torch.randn(*s, generator=gen)
    x, gamma, c, vx, vg = rand(m, heads, d), 1 + 0.3 * rand(d), rand(m, heads, d), rand(m, heads, d), rand(d)
    table = L.loract_rope_table(m, d)
    f = lambda e: L.loract_qknorm_rope_forward((x + e * vx).cuda(), None, (gamma + e * vg).cuda(), None, table, interleaved=interleaved)[0].double()
    num = ((f(h) - f(-h)) * c.cuda().double()).sum().item() / (2 * h)
    dx, _, dg, _ = L.loract_qknorm_rope_backward(x.cuda(), None, gamma.cuda(), None, table, c.cuda(), None, interleaved=interleaved)
    ana = (dx.cpu().double() * vx.double()).sum().item() + (dg.cpu().double() * vg.double()).sum().item()
    size = math.sqrt(m * heads * d) * (h * h * 8 + 2.0 ** -22 * 4 / h) * 6
    assert abs(num - ana) <= size, (num, ana, size)
