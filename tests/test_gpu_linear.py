"""loract_linear and loract_linear_backward against plain 64-bit arithmetic."""
import math

import pytest
import torch

import sublayer_ref as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rand(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def _strided(t, pad, shift):
    """The same matrix on the GPU as a slice of a larger one: row pitch + pad, first element `shift` elements in."""
    big = torch.full((t.shape[0], t.shape[1] + pad + shift), float("nan"), dtype=t.dtype, device="cuda")
    view = big[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view


def _case(m, n_in, n_out, dtype="bf16", layout="nt", act="none", bias=False, r=0, p=0.0, residual=False, keep=False,
          out_dtype=None, pad=0, shift=0, seed=1, poison=None):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    odt = DT[out_dtype or dtype]
    x, w = _rand(gen, m, n_in, dtype=dt), _rand(gen, n_out, n_in, dtype=dt, scale=n_in ** -0.5)
    if poison:
        poison(x, w)
    b = _rand(gen, n_out) if bias else None
    t = _rand(gen, m, r, dtype=dt) if r else None
    lb = _rand(gen, r, n_out, dtype=dt, scale=0.3) if r else None
    res = _rand(gen, m, n_out, dtype=dt) if residual else None
    fac = ref.drop_factors(m, n_out, p, 77 + seed) if p else None
    d = lambda v: None if v is None else v.double()
    y, pre, perr = ref.linear(x.double(), w.double(), d(b), d(t), d(lb), -0.75, act, fac, d(res))
    g = lambda v: None if v is None else v.cuda()
    wl = w if layout == "nt" else w.t().contiguous()
    out = torch.full((m, n_out + pad), float("nan"), dtype=odt, device="cuda")[:, :n_out] if pad else None
    got = L.loract_linear(_strided(x, pad, shift), _strided(wl, pad, shift), g(b), w_transposed=layout == "nn", lora_t=g(t), lora_b=g(lb),
                          lora_scale=-0.75, act=act, p_drop=p, seed=77 + seed, residual=None if res is None else _strided(res, pad, shift),
                          save_preact=keep, out_dtype=odt, out=out)
    z = None
    if keep:
        got, z = got
    assert got.dtype == odt
    ref.check(got, y, ref.linear_bound(y, pre, perr, odt, fac, d(res)), "Y")
    if keep:
        assert z.dtype == dt
        ref.check(z, pre, perr + 1.01 * ref.U[dt] * (pre.abs() + perr), "Z")
    return got


SIZES = [(1, 1, 1), (1, 8, 5), (2, 64, 64), (3, 7, 130), (16, 512, 100), (17, 65, 16), (33, 96, 300), (64, 128, 64), (65, 72, 257),
         (128, 64, 128), (129, 200, 129), (200, 1032, 40), (300, 320, 512), (5, 2056, 7), (260, 33, 520), (513, 256, 1030),
         (1, 4096, 512), (4, 1000, 3000), (40, 3000, 48), (1025, 64, 4), (700, 136, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out", SIZES)
def test_product(m, n_in, n_out, layout, dtype):
    _case(m, n_in, n_out, dtype=dtype, layout=layout)


# many tiles: K of one slab and of several, whole and ragged, edges in both directions
@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out,parts", [
    (2816, 128, 3080, dict()), (2817, 136, 2824, dict(keep=True)), (4000, 200, 2048, dict(r=16, act="silu", bias=True, keep=True)),
    (2900, 264, 2816, dict(r=33, p=0.1, residual=True)), (8, 64, 64, dict()), (3000, 168, 3000, dict(r=64, act="gelu", out_dtype="f32")),
    (2818, 520, 2832, dict(r=8, act="relu", bias=True, p=0.2, residual=True, keep=True)), (33000, 192, 256, dict(r=5)),
    (260, 448, 33000, dict(r=40, residual=True)), (3001, 1000, 2808, dict(p=0.3)), (2816, 384, 2816, dict(pad=8, shift=8, r=16, residual=True)),
    (2816, 152, 2816, dict(pad=24, shift=16, r=12, act="gelu", bias=True, p=0.1))])
def test_large_tiles(m, n_in, n_out, parts, layout):
    _case(m, n_in, n_out, layout=layout, **parts)


# 256 tiles of 256 x 256, the smaller tiles with K split and whole, edges in both directions
@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out,parts", [
    (3900, 136, 4088, dict(keep=True)), (4096, 200, 4096, dict(r=16, act="silu", bias=True, keep=True)), (3841, 264, 3848, dict(r=33, p=0.1, residual=True)),
    (4000, 456, 3992, dict(r=64, act="gelu", out_dtype="f32")), (65536, 64, 256, dict(r=40, act="relu", bias=True)), (256, 328, 65536, dict(p=0.2, residual=True)),
    (4090, 72, 4000, dict(pad=8, shift=8, r=12, residual=True)), (65, 2056, 72, dict(r=16, act="silu", bias=True, keep=True)),
    (300, 2400, 200, dict(residual=True, p=0.1)), (127, 8192, 136, dict(r=33, out_dtype="f32")), (129, 1096, 264, dict(act="gelu")),
    (70, 64, 80, dict(r=64)), (1000, 648, 520, dict(pad=16, shift=8, r=8, residual=True)), (66, 4168, 4096, dict(keep=True, r=5)),
    (2000, 128, 1000, dict(p=0.1)), (333, 1480, 408, dict(bias=True))])
def test_both_tiles(m, n_in, n_out, parts, layout):
    _case(m, n_in, n_out, layout=layout, **parts)


# few tokens, few outputs: K that fills no wave's share, one and two blocks of 16, several workgroups along K
@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out,parts", [
    (1, 8, 8, dict()), (1, 40, 24, dict(r=3)), (1, 4104, 136, dict(r=64, act="silu", bias=True, keep=True)), (7, 2048, 264, dict(r=33, residual=True)),
    (16, 264, 1000, dict(p=0.2, act="gelu")), (17, 1032, 520, dict(r=16, keep=True)), (32, 72, 4096, dict(r=8, residual=True, p=0.1)),
    (32, 11008, 40, dict(out_dtype="f32", act="relu")), (5, 8200, 64, dict(residual=True, keep=True, r=40)), (2, 32, 5, dict()),
    (300, 264, 16, dict(r=16)), (300, 8, 64, dict(residual=True)), (333, 2056, 8, dict(act="silu", bias=True)), (9000, 104, 16, dict(r=7, p=0.1)),
    (8200, 256, 48, dict(keep=True, act="gelu", r=64)), (100, 4096, 33, dict(bias=True)), (70, 8192, 24, dict(pad=8, shift=8, residual=True)),
    (4, 512, 128, dict(pad=16, shift=8, r=12, act="silu", keep=True))])
def test_thin_products(m, n_in, n_out, parts, layout):
    _case(m, n_in, n_out, layout=layout, **parts)


@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out,parts", [
    (1, 8, 4, dict()), (1, 9, 12, dict(r=3)), (1, 4101, 132, dict(r=64, act="silu", bias=True, keep=True)), (7, 1027, 260, dict(r=33, residual=True)),
    (16, 260, 1000, dict(p=0.2, act="gelu")), (17, 517, 516, dict(r=16, keep=True)), (32, 72, 4096, dict(r=8, residual=True, p=0.1)),
    (32, 5003, 44, dict(act="relu", r=48)), (2, 32, 5, dict()), (300, 267, 16, dict(r=16)), (333, 1031, 8, dict(act="silu", bias=True)),
    (9000, 101, 28, dict(r=7, p=0.1)), (8200, 256, 32, dict(keep=True, act="gelu", r=64)), (70, 4099, 20, dict(pad=4, shift=8, residual=True)),
    (100, 640, 17, dict(pad=3, shift=1, r=5)), (4, 512, 128, dict(pad=12, shift=4, r=12, act="silu", keep=True))])
def test_thin_products_of_float32(m, n_in, n_out, parts, layout):
    _case(m, n_in, n_out, dtype="f32", layout=layout, **parts)


def test_large_tiles_keep_nan_and_infinity_where_they_belong():
    for layout in ("nt", "nn"):
        def poison(x, w):
            x[17, 199] = float("nan")
            w[2815, 0] = float("inf")
            x[:, 0] = x[:, 0].abs() + 0.5
        got = _case(2816, 200, 2816, layout=layout, poison=poison).float().cpu()
        bad = ~torch.isfinite(got)
        assert bad[17].all() and bad[:, 2815].all() and int(bad.sum()) == 2816 * 2 - 1
        got = _case(3900, 200, 4096, layout=layout, poison=poison).float().cpu()
        bad = ~torch.isfinite(got)
        assert bad[17].all() and bad[:, 2815].all() and int(bad.sum()) == 3900 + 4096 - 1


@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("dtype,out_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,n_in,n_out,r", [(1, 64, 96, 4), (19, 136, 67, 33), (150, 264, 260, 16), (257, 512, 384, 64), (8, 768, 1024, 8)])
def test_epilogue(m, n_in, n_out, r, act, dtype, out_dtype, layout):
    _case(m, n_in, n_out, dtype=dtype, out_dtype=out_dtype, layout=layout, act=act, bias=True, r=r, p=0.25, residual=True, keep=True)


@pytest.mark.parametrize("parts", [dict(bias=True), dict(r=1), dict(r=64), dict(p=0.5), dict(residual=True), dict(keep=True, act="silu"),
                                   dict(r=40, residual=True), dict(p=0.99999), dict(p=1e-6)])
@pytest.mark.parametrize("m,n_in,n_out", [(2, 128, 192), (140, 192, 256), (300, 576, 24)])
def test_parts_of_the_epilogue(m, n_in, n_out, parts):
    _case(m, n_in, n_out, **parts)
    _case(m, n_in, n_out, layout="nn", **parts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 1), (4, 4), (1, 0)])
@pytest.mark.parametrize("m,n_in,n_out", [(3, 256, 96), (300, 320, 272), (130, 512, 16)])
def test_strides_and_alignment(m, n_in, n_out, pad, shift, layout, dtype):
    _case(m, n_in, n_out, dtype=dtype, layout=layout, pad=pad, shift=shift, residual=True, p=0.1, r=8, bias=True, act="gelu")


@pytest.mark.parametrize("layout", ["nt", "nn"])
@pytest.mark.parametrize("m,n_in,n_out", [(2, 600, 64), (300, 1000, 300), (257, 512, 24)])
def test_nan_and_infinity_stay_where_they_belong(m, n_in, n_out, layout):
    def poison(x, w):
        x[m // 2, n_in - 1] = float("nan")
        w[n_out - 1, 0] = float("inf")
        x[:, 0] = x[:, 0].abs() + 0.5                  # (the infinity gets one sign)
    got = _case(m, n_in, n_out, layout=layout, poison=poison).float().cpu()
    bad = ~torch.isfinite(got)
    want = torch.zeros_like(bad)
    want[m // 2] = True
    want[:, n_out - 1] = True
    assert torch.equal(bad, want)


def test_dropped_places_hide_whatever_was_there():
    import paper_2509_23472_amd as L
    m, n = 64, 256
    x = torch.full((m, 64), float("inf"), dtype=torch.bfloat16, device="cuda")
    w = torch.ones((n, 64), dtype=torch.bfloat16, device="cuda")
    y = L.loract_linear(x, w, p_drop=0.5, seed=9).float().cpu()
    keep = ref.drop_factors(m, n, 0.5, 9) > 0
    assert (y[~keep] == 0).all() and torch.isinf(y[keep]).all()
    dp, _, _ = L.loract_linear_backward(torch.full((m, n), float("nan"), device="cuda"), p_drop=0.5, seed=9)
    assert (dp.cpu()[~keep] == 0).all() and torch.isnan(dp.cpu()[keep]).all()


def test_operands_that_do_not_fit_are_refused():
    import paper_2509_23472_amd as L
    x, w = torch.zeros((8, 64), device="cuda"), torch.zeros((32, 64), device="cuda")
    t, b = torch.zeros((8, 4), device="cuda"), torch.zeros((4, 32), device="cuda")
    calls = [lambda: L.loract_linear(x, w.bfloat16()), lambda: L.loract_linear(x, w, w_transposed=True), lambda: L.loract_linear(x, w, lora_t=t),
             lambda: L.loract_linear(x, w, lora_t=t, lora_b=b[:3]), lambda: L.loract_linear(x, w, torch.zeros(31, device="cuda")),
             lambda: L.loract_linear(x, w, torch.zeros(32, device="cuda").half()), lambda: L.loract_linear(x, w, residual=x), lambda: L.loract_linear(x, w, act="tanh"),
             lambda: L.loract_linear(x, w, out=torch.zeros((8, 1), device="cuda").expand(8, 32)), lambda: L.loract_linear(x.t(), w), lambda: L.loract_linear(x[0], w),
             lambda: L.loract_linear_backward(x, act="silu"), lambda: L.loract_linear_backward(x, x[:4], act="silu"), lambda: L.loract_linear_backward(x, lora_t=t[:4]),
             lambda: L.loract_dropout(x, 0.1, 0, residual=w), lambda: L.loract_dropout(x[:1].expand(8, 64), 0.1, 0)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: L.loract_linear(x, w, p_drop=1.0), lambda: L.loract_dropout(x, -0.5, 0), lambda: L.loract_linear(x, w, out_dtype=torch.bfloat16),
                 lambda: L.loract_linear(x, w, lora_t=torch.zeros((8, 65), device="cuda"), lora_b=torch.zeros((65, 32), device="cuda"))):
        with pytest.raises(L.LoractError):
            call()
    with pytest.raises(TypeError):
        L.loract_linear(x.half(), w.half())


def test_calls_can_be_captured_and_replayed():
    """Nothing is enqueued but kernels, and every replay gives what the call gives, with other work in between."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(9)
    x, w, wt = (_rand(gen, *s, dtype=torch.bfloat16).cuda() for s in ((300, 512), (256, 512), (512, 24)))
    lt = _rand(gen, 300, 8, dtype=torch.bfloat16).cuda()
    lb = _rand(gen, 8, 256, dtype=torch.bfloat16).cuda()
    table, gamma = L.loract_rope_table(300, 64), torch.ones(64, device="cuda")

    def work():
        y, z = L.loract_linear(x, w, lora_t=lt, lora_b=lb, act="gelu", p_drop=0.1, seed=3, save_preact=True)
        t = L.loract_linear(x, wt, w_transposed=True)
        back = L.loract_linear_backward(y, z, lora_t=lt, act="gelu", p_drop=0.1, seed=3)
        heads = y.view(300, 4, 64)
        return (y, z, t) + back + L.loract_qknorm_rope_backward(heads, None, gamma, None, table, heads, None)[::2] + (L.loract_dropout(y, 0.5, 1),)

    want = [v.clone() for v in work()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        work()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = work()
    for _ in range(4):
        for v in got:
            v.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.randn(1000, 1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")


def test_no_tokens():
    import paper_2509_23472_amd as L
    x, w = torch.zeros((0, 64), device="cuda"), torch.zeros((32, 64), device="cuda")
    assert L.loract_linear(x, w).shape == (0, 32)
    dp, db, d_b = L.loract_linear_backward(torch.zeros((0, 32), device="cuda"), lora_t=torch.zeros((0, 4), device="cuda"))
    assert dp.shape == (0, 32) and not db.any() and d_b.shape == (4, 32) and not d_b.any()


def test_offsets_past_32_bits():
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(3)
    m, k, n, pitch = 2100, 64, 96, 1 << 20
    x, w = _rand(gen, m, k, dtype=torch.bfloat16), _rand(gen, n, k, dtype=torch.bfloat16)
    xb = torch.empty((m, pitch), dtype=torch.bfloat16, device="cuda")[:, :k]
    xb.copy_(x)
    yb = torch.empty((m, pitch), dtype=torch.bfloat16, device="cuda")[:, pitch - n:]
    L.loract_linear(xb, w.cuda(), out=yb)
    y, pre, perr = ref.linear(x.double(), w.double())
    ref.check(yb, y, ref.linear_bound(y, pre, perr, torch.bfloat16), "Y")
    wt = torch.empty((k, 1 << 26), dtype=torch.bfloat16, device="cuda")[:, :n]          # 64 rows, 2^32 elements apart in all
    wt.copy_(w.t())
    got = L.loract_linear(x.cuda(), wt, w_transposed=True)
    ref.check(got, y, ref.linear_bound(y, pre, perr, torch.bfloat16), "Y from transposed weights")


@pytest.mark.parametrize("m,n_in,n_out", [(1, 4096, 512), (300, 1024, 256), (513, 2048, 16)])
def test_in_place_residual_side_stream_and_repetition(m, n_in, n_out):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(5)
    x, w = _rand(gen, m, n_in, dtype=torch.bfloat16).cuda(), _rand(gen, n_out, n_in, dtype=torch.bfloat16).cuda()
    res = _rand(gen, m, n_out, dtype=torch.bfloat16).cuda()
    first = L.loract_linear(x, w, residual=res, p_drop=0.2, seed=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = L.loract_linear(x, w, residual=res, p_drop=0.2, seed=4)
    side.synchronize()
    assert torch.equal(first, again)
    L.loract_linear(x, w, residual=res, p_drop=0.2, seed=4, out=res)
    assert torch.equal(first, res)


# ---------------------------------------------------------------------------------------------
# Backward.

def _back(m, n, dtype="bf16", act="none", r=0, p=0.0, bias=True, pad=0, shift=0, seed=1):
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    dy, z = _rand(gen, m, n, dtype=dt), _rand(gen, m, n, dtype=dt, scale=2.0)
    t = _rand(gen, m, r, dtype=dt) if r else None
    fac = ref.drop_factors(m, n, p, 31 + seed)
    sl = ref.slope(act, z.double())
    want = dy.double() * fac * sl
    out = torch.full((m, n + pad), float("nan"), dtype=dt, device="cuda")[:, :n] if pad else None
    dp, db, d_b = L.loract_linear_backward(_strided(dy, pad, shift), _strided(z, pad, shift) if act != "none" else None,
                                           lora_t=None if t is None else t.cuda(), lora_scale=0.5, act=act, p_drop=p, seed=31 + seed,
                                           bias_grad=bias, out=out)
    # a slope is a sum of terms up to 1 + |z| in size, each a few roundings off
    err = (dy.double() * fac).abs() * 16 * 2.0 ** -24 * (1 + (z.double().abs() if act != "none" else 0)) + 2.0 ** -23 * want.abs()
    ref.check(dp, want, err + 1.01 * ref.U[dt] * (want.abs() + err) + 1e-37, "dP")
    many = 6 * math.sqrt(m) * 2.0 ** -24
    if bias:
        ref.check(db, want.sum(0), err.sum(0) + many * want.abs().sum(0), "db")
    else:
        assert db is None
    if r:
        mag = t.double().abs().t() @ want.abs()
        ref.check(d_b, 0.5 * (t.double().t() @ want), 0.5 * (t.double().abs().t() @ err) + many * mag + 2.0 ** -23 * mag, "dB")
    else:
        assert d_b is None
    return dp, db, d_b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("r", [0, 1, 16, 17, 48, 64])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 128), (3, 130), (70, 64), (129, 257), (500, 40), (1000, 200)])
def test_backward(m, n, r, act, dtype):
    _back(m, n, dtype=dtype, act=act, r=r, p=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("parts", [dict(bias=False), dict(bias=False, r=5), dict(p=0.0, r=8), dict(pad=8, r=3, act="silu"),
                                   dict(pad=3, shift=1, r=9, act="gelu", p=0.1), dict(pad=1, act="relu")])
@pytest.mark.parametrize("m,n", [(5, 96), (300, 264), (2100, 72)])
def test_backward_parts_and_strides(m, n, parts, dtype):
    _back(m, n, dtype=dtype, **parts)


def test_backward_repeats_bit_for_bit_and_in_place():
    import paper_2509_23472_amd as L
    a, b = _back(1000, 264, act="gelu", r=16, p=0.1), _back(1000, 264, act="gelu", r=16, p=0.1)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    dy = torch.randn(100, 64, device="cuda")
    want, _, _ = L.loract_linear_backward(dy, p_drop=0.4, seed=2)
    got, _, _ = L.loract_linear_backward(dy, p_drop=0.4, seed=2, out=dy)
    assert got.data_ptr() == dy.data_ptr() and torch.equal(got, want)


def test_slopes_at_the_ends_of_the_range():
    import paper_2509_23472_amd as L
    z = torch.tensor([[-3e38, -1e4, -200.0, -90.0, -20.0, -0.0, 0.0, 20.0, 90.0, 200.0, 1e4, 3e38]], device="cuda")
    for act in ("relu", "gelu", "silu"):
        dp, _, _ = L.loract_linear_backward(torch.ones_like(z), z, act=act)
        want = ref.slope(act, z.double().cpu())
        ref.check(dp, want, 1e-6 * torch.ones_like(want), act)
        x, w = z.t().contiguous(), torch.ones((1, 1), device="cuda")
        y = L.loract_linear(x, w, act=act)
        want = ref.act(act, x.double().cpu())
        ref.check(y, want, 1e-6 * want.abs() + 1e-6, act)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_gradients_against_differences(act):
    """d/dh of sum C Y(X + h dX, bias + h db, B + h dB) against the gradients' products with the directions.

    float32 throughout; the difference at h = 2^-6 is off by h^2 / 6 times a third derivative of order 1 for
    every output, and by the outputs' rounding, 2^-22 |Y| / h for each of them, both at random signs."""
    import paper_2509_23472_amd as L
    gen = torch.Generator().manual_seed(11)
    m, k, n, r, h, p = 48, 40, 56, 8, 2.0 ** -6, 0.2
    rand = lambda *s: torch.randn(*s, generator=gen)
    x, w, bias, a, b, c = rand(m, k), rand(n, k) / k ** 0.5, rand(n), rand(k, r) / k ** 0.5, rand(r, n) / r ** 0.5, rand(m, n)
    if act == "relu":                                   # no element near the kink
        c = torch.where((ref.linear(x.double(), w.double(), bias.double(), (x @ a).double(), b.double(), 0.5)[1]).abs() < 0.3, torch.zeros_like(c), c)
    dx, dbias, da, db = rand(m, k), rand(n), rand(k, r) / k ** 0.5, rand(r, n) / r ** 0.5
    g = lambda v: v.contiguous().cuda()

    def forward(e, keep=False):
        xe, ae = g(x + e * dx), g(a + e * da)
        t = L.loract_linear(xe, ae, w_transposed=True)
        return L.loract_linear(xe, g(w), g(bias + e * dbias), lora_t=t, lora_b=g(b + e * db), lora_scale=0.5, act=act, p_drop=p, seed=3,
                               save_preact=keep), t

    (y, z), t = forward(0.0, True)
    num = ((forward(h)[0].double() - forward(-h)[0].double()) * c.cuda().double()).sum().item() / (2 * h)
    dp, g_bias, g_b = L.loract_linear_backward(g(c), z, lora_t=t, lora_scale=0.5, act=act, p_drop=p, seed=3)
    g_t = L.loract_linear(dp, g(b)) * 0.5                                   # dT = s dP B^T
    g_x = L.loract_linear(dp, g(w), w_transposed=True, lora_t=g_t, lora_b=g(a.t()))
    g_a = x.cuda().double().t() @ g_t.double()
    ana = sum((u.double().cpu() * v.double()).sum().item() for u, v in ((g_x, dx), (g_bias, dbias), (g_b, db), (g_a, da)))
    size = math.sqrt(m * n) * (h * h * 8 + 2.0 ** -22 * 4 / h) * 6
    assert abs(num - ana) <= size, (num, ana, size)
